// fs_attention.hip -- causal attention over the paged 8-bit cache.
//
// o_i = sum_j softmax_j(scale <q_i, K_j>) V_j with K_j = kscale * kcode_j and
// V_j = vscale * vcode_j.  One pass over the tokens with the running maximum
// and sum; the context is split over blocks when there are few rows, and a
// second kernel joins the parts.
#include "fs_serving.h"

namespace fs {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kFloor = -1e30f;  // a maximum over no tokens: finite, so differences stay numbers
constexpr int kTile = 64;         // tokens of one step of a wavefront

// ------------------------------------------------------------ the work list --
// Work items: (sequence, tile of R rows, cache head, part of the context).
// A row is a (new token, query head of the group) pair of one cache head.
// Each block derives the same list from the lengths alone.

struct Seq {
  int q0, n;         // first row of q, new tokens
  int length;        // tokens in the cache
  int t0, t1;        // 64-token tiles that some query sees
};

__device__ __forceinline__ Seq sequence(const AttendArgs &A, int s) {
  Seq q;
  q.q0 = min(max(A.cu_q[s], 0), A.n_tokens);
  q.n = min(max(A.cu_q[s + 1], q.q0), A.n_tokens) - q.q0;
  const int64_t room = min(A.table_width << A.c.page_shift, (int64_t)0x7fffffc0);
  q.length = (int)min((int64_t)max(A.ctx_lens[s], 0), room);
  const int64_t first = (int64_t)q.length - q.n;
  const int64_t from = A.window ? max((int64_t)0, first - A.window + 1) : 0;
  q.t0 = (int)(from / kTile);
  q.t1 = q.n ? (int)(((int64_t)q.length + kTile - 1) / kTile) : q.t0;
  return q;
}

struct List {
  int items, partials;  // items in all; those of split contexts
  int chunk;            // tiles an item has at most
};

__device__ __forceinline__ int row_tiles(const Seq &q, int group, int R) { return (int)(((int64_t)q.n * group + R - 1) / R); }
__device__ __forceinline__ int parts_of(const Seq &q, int chunk) { return max(1, (q.t1 - q.t0 + chunk - 1) / chunk); }

// Prefix sums over the sequences of items (pre) and of items of split
// contexts (part), in LDS; all threads of the block call it.
template <int THREADS, int R>
__device__ List make_list(const AttendArgs &A, int group, int target, int least, int *pre, int *part) {
  __shared__ int64_t work[THREADS / 64];
  __shared__ int2 carry[THREADS / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t heads = A.c.n_heads;
  int64_t w = 0;
  for (int s = threadIdx.x; s < A.n_seqs; s += THREADS) {
    const Seq q = sequence(A, s);
    w += heads * row_tiles(q, group, R) * (q.t1 - q.t0);
  }
  for (int o = 32; o; o >>= 1) w += __shfl_xor(w, o);
  if (lane == 0) work[wave] = w;
  __syncthreads();
  w = 0;
  for (int i = 0; i < THREADS / 64; ++i) w += work[i];
  List L;
  L.chunk = (int)min(max((w + target - 1) / target, (int64_t)least), (int64_t)0x3fffffff);
  int2 base = {0, 0};
  for (int s0 = 0; s0 < A.n_seqs; s0 += THREADS) {
    const int s = s0 + threadIdx.x;
    int2 v = {0, 0};
    if (s < A.n_seqs) {
      const Seq q = sequence(A, s);
      const int parts = parts_of(q, L.chunk);
      v.x = (int)heads * row_tiles(q, group, R) * parts;
      v.y = parts > 1 ? v.x : 0;
    }
    int2 sum = v;
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(sum.x, o), y = __shfl_up(sum.y, o);
      if (lane >= o) {
        sum.x += x;
        sum.y += y;
      }
    }
    if (lane == 63) carry[wave] = sum;
    __syncthreads();
    int2 before = base;
    for (int i = 0; i < THREADS / 64; ++i) {
      if (i < wave) {
        before.x += carry[i].x;
        before.y += carry[i].y;
      }
      base.x += carry[i].x;
      base.y += carry[i].y;
    }
    if (s < A.n_seqs) {
      pre[s] = before.x + sum.x - v.x;
      part[s] = before.y + sum.y - v.y;
    }
    __syncthreads();
  }
  L.items = base.x;
  L.partials = base.y;
  return L;
}

// The last sequence whose prefix is at most `item` (one with items: those
// without share their prefix with the next).
__device__ __forceinline__ int find(const int *prefix, int n, int item) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (prefix[mid] <= item) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The tiles of part `ch` of `parts` of the tokens that rows r0 .. r1 - 1 see.
__device__ __forceinline__ int2 tiles_of(const AttendArgs &A, const Seq &q, int group, int r0, int r1, int parts, int ch) {
  const int64_t first = (int64_t)q.length - q.n;
  const int64_t j0 = r0 / group, j1 = min((int64_t)q.n - 1, (int64_t)(r1 - 1) / group);
  const int64_t end = min((int64_t)q.length, first + j1 + 1);
  const int64_t from = A.window ? max((int64_t)0, first + j0 - A.window + 1) : 0;
  if (end <= from) return {0, 0};
  const int a = (int)(from / kTile), b = (int)((end + kTile - 1) / kTile);
  const int len = (b - a + parts - 1) / parts;
  return {min(b, a + ch * len), min(b, a + (ch + 1) * len)};
}

// Workspace: per part of a split context the rows' maximum and sum, then
// their unnormalised outputs.
constexpr int kRows = 16;
__host__ __device__ constexpr int64_t part_floats(int R, int D) { return (int64_t)R * (D + 2); }

// --------------------------------------------------- rows by 16, 8-bit products --
// One wavefront takes 64 tokens of the context at a time for 16 rows.
//
// Keys and values stay 8-bit integers: q = (256 hi + lo) * step with 15-bit
// codes against the row's largest magnitude, two exact integer products make
// S; the probabilities of a tile, against its largest, are 15-bit codes too.
// S^T = K Q^T leaves a lane with one row and 16 tokens, and with the tokens
// of the four S tiles dealt as G*16 + t*4 + i (G = lane / 16) those 16 are
// neighbours: packed to bytes they are the second operand of O^T = V^T P^T as
// they stand, and a lane's piece of V^T is one 16-byte load.  A page's value
// scale is added to the exponent (log2), so one tile may span pages; the sum
// of the softmax is kept in binary32 without it.

template <int TYPE, int D>
__global__ __launch_bounds__(256) void k_attend_rows(AttendArgs A, int target, int least, float *ws) {
  constexpr int STEPS = D / 64, DT = D / 16;
  extern __shared__ int dynamic[];
  int *const pre = dynamic, *const part = dynamic + A.n_seqs;
  __shared__ float lo[4][kRows][D + 4];
  __shared__ float lm[4][kRows], ll[4][kRows];
  const Cache &c = A.c;
  const int group = A.n_q_heads / c.n_heads;
  const List L = make_list<256, kRows>(A, group, target, least, pre, part);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = lane & 15, G = lane >> 4, kg = row >> 2;
  const int PS = 1 << c.page_shift;

  for (int item = blockIdx.x; item < L.items; item += gridDim.x) {
    const int s = find(pre, A.n_seqs, item);
    const Seq q = sequence(A, s);
    const int parts = parts_of(q, L.chunk);
    int at = item - pre[s];
    const int ch = at % parts;
    at /= parts;
    const int h = at % c.n_heads, r0 = at / c.n_heads * kRows, rows = min(kRows, q.n * group - r0);
    const int2 span = tiles_of(A, q, group, r0, r0 + rows, parts, ch);
    const int first = q.length - q.n;
    const int r = r0 + row, token = row < rows ? r / group : 0;
    const int64_t q_row = q.q0 + token;
    const int q_head = h * group + r % group;
    // what this row sees
    const int last_seen = row < rows ? first + token : -1;
    const int first_seen = A.window ? max(0, last_seen - A.window + 1) : 0;
    // pages that some row of the tile sees
    const int top = first + min(q.n - 1, (r0 + rows - 1) / group);
    const int low = A.window ? max(0, first + r0 / group - A.window + 1) : 0;
    const int page_top = max(top, 0) >> c.page_shift, page_low = min(low, max(top, 0)) >> c.page_shift;

    // the row's codes
    float x[STEPS][16];
    uint32_t most = 0;
    for (int st = 0; st < STEPS; ++st) {
      uint16_t raw[16] = {};
      if (row < rows)
        __builtin_memcpy(raw, (const uint16_t *)A.q + q_row * A.q_stride + q_head * D + st * 64 + G * 16, 32);
      for (int i = 0; i < 16; ++i) {
        x[st][i] = value16<TYPE>(raw[i]);
        most = max(most, __float_as_uint(x[st][i]) & 0x7fffffffu);
      }
    }
    most = max(most, (uint32_t)__shfl_xor((int)most, 16));
    most = max(most, (uint32_t)__shfl_xor((int)most, 32));
    const float largest = __uint_as_float(most);
    const float inverse = largest < kTiny ? 0.0f : 32512.0f / largest;
    const float q_step = (largest < kTiny ? 0.0f : largest / 32512.0f) * (A.scale * kLog2e);
    int4v q_hi[STEPS], q_lo[STEPS];
    for (int st = 0; st < STEPS; ++st)
      for (int w = 0; w < 4; ++w) {
        uint32_t hi = 0, low_bytes = 0;
        for (int i = 0; i < 4; ++i) {
          const int v = (int)rintf(x[st][w * 4 + i] * inverse);
          hi |= (uint32_t)(((v + 128) >> 8) & 0xff) << (8 * i);
          low_bytes |= (uint32_t)(v & 0xff) << (8 * i);  // v - 256 * ((v + 128) >> 8), as a signed byte
        }
        q_hi[st][w] = (int)hi;
        q_lo[st][w] = (int)low_bytes;
      }

    float4v o[DT] = {};
    float m = kFloor, l = 0.0f;
    const int32_t *const table = A.table + s * A.table_width;
    for (int tile = span.x + wave; tile < span.y; tile += 4) {
      const int base = tile * kTile;
      const auto page_of = [&](int tok) {
        const int i = min(max(tok >> c.page_shift, page_low), page_top);
        return (int64_t)min((uint32_t)table[i], (uint32_t)(c.n_pages - 1)) * c.n_heads + h;
      };
      const int64_t pk = page_of(base + kg * 16), pv = page_of(base + G * 16);
      const int8_t *const kp = c.k + (pk * PS + ((base + kg * 16) & (PS - 1)) + (row & 3)) * D + G * 16;
      const int8_t *const vp = c.v + (pv * D + row) * PS + ((base + G * 16) & (PS - 1));
      int4v kf[4][STEPS], vf[DT];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int st = 0; st < STEPS; ++st) kf[t][st] = *(const int4v *)(kp + t * 4 * D + st * 64);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) vf[dt] = *(const int4v *)(vp + dt * 16 * PS);
      float ks = c.k_scale[pk - pk + pv], vs = c.v_scale[pv];
      // tokens of this lane that the row sees: base + G*16 + [a, b]
      const int mine = base + G * 16;
      const bool all = base >= first_seen && base + kTile - 1 <= last_seen;
      const bool masked = __any(!all);
      if (masked && (last_seen < mine || first_seen > mine + 15)) ks = vs = 1.0f;  // no page of this row's
      const bool zero = vs < kZeroScale;
      const float lift = zero ? -60.0f : __builtin_amdgcn_logf(vs);
      const float per = zero ? 0x1p60f : 1.0f / vs;
      const float cq = q_step * ks;
      float sc[16];
      float top_s = kFloor;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        int4v hi = {0, 0, 0, 0}, low_sum = {0, 0, 0, 0};
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf[t][st], q_hi[st], hi, 0, 0, 0);
          low_sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf[t][st], q_lo[st], low_sum, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v = __builtin_fmaf((float)(hi[i] * 256 + low_sum[i]), cq, lift);
          if (masked) {
            const int tok = mine + t * 4 + i;
            v = tok >= first_seen && tok <= last_seen ? v : -INFINITY;
          }
          sc[t * 4 + i] = v;
          top_s = fmaxf(top_s, v);
        }
      }
      top_s = fmaxf(top_s, __shfl_xor(top_s, 16));
      top_s = fmaxf(top_s, __shfl_xor(top_s, 32));
      const float m_new = fmaxf(m, top_s);
      const float keep = __builtin_amdgcn_exp2f(m - m_new), add = __builtin_amdgcn_exp2f(top_s - m_new);
      m = m_new;
      // probabilities against the tile's largest: 15-bit codes, in the low
      // bits of a sum with 2^23 + 128 (the 128 makes the low byte signed)
      const float full = zero ? 0.0f : 32512.0f;
      float sum = 0.0f;
      int4v p_hi, p_lo;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = __builtin_amdgcn_exp2f(sc[t * 4 + i] - top_s);
          sum += p;
          b[i] = __float_as_uint(__builtin_fmaf(p, full, 8388608.0f + 128.0f));
        }
        const uint32_t u = __builtin_amdgcn_perm(b[1], b[0], 0x05010400), v = __builtin_amdgcn_perm(b[3], b[2], 0x05010400);
        p_lo[t] = (int)(__builtin_amdgcn_perm(v, u, 0x05040100) ^ 0x80808080u);
        p_hi[t] = (int)__builtin_amdgcn_perm(v, u, 0x07060302);
      }
      l = l * keep + sum * per * add;
      const float step = add * (1.0f / 32512.0f);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const int4v none = {0, 0, 0, 0};
        const int4v hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(vf[dt], p_hi, none, 0, 0, 0);
        const int4v low_sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(vf[dt], p_lo, none, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          o[dt][i] = __builtin_fmaf((float)(hi[i] * 256 + low_sum[i]), step, o[dt][i] * keep);
      }
    }
    // the row's sum over the four lanes that hold it, then the four wavefronts
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (G == 0) {
      lm[wave][row] = m;
      ll[wave][row] = l;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *(float4v *)&lo[wave][row][dt * 16 + G * 4] = o[dt];
    __syncthreads();
    for (int e = threadIdx.x; e < rows * D; e += 256) {
      const int i = e / D, d = e % D;
      float M = lm[0][i];
      for (int w = 1; w < 4; ++w) M = fmaxf(M, lm[w][i]);
      float sum = 0.0f, out = 0.0f;
      for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f(lm[w][i] - M);
        sum += f * ll[w][i];
        out += f * lo[w][i][d];
      }
      if (parts > 1) {
        float *const to = ws + (part[s] + item - pre[s]) * part_floats(kRows, D);
        if (d == 0) {
          to[i] = M;
          to[kRows + i] = sum;
        }
        to[2 * kRows + i * D + d] = out;
      } else {
        const int rr = r0 + i;
        store_value<TYPE>(A.out, ((int64_t)(q.q0 + rr / group) * A.n_q_heads + h * group + rr % group) * D + d,
                          sum == 0.0f ? 0.0f : out / sum);
      }
    }
    __syncthreads();
  }
}

// Joins the parts of split contexts: a block takes one row tile of one head.
template <int TYPE, int D, int R>
__global__ __launch_bounds__(256) void k_join(AttendArgs A, int target, int least, const float *ws) {
  extern __shared__ int dynamic[];
  int *const pre = dynamic, *const part = dynamic + A.n_seqs;
  const int group = A.n_q_heads / A.c.n_heads;
  const List L = make_list<256, R>(A, group, target, least, pre, part);
  for (int at = blockIdx.x; at < L.partials; at += gridDim.x) {
    const int s = find(part, A.n_seqs, at);
    const Seq q = sequence(A, s);
    const int parts = parts_of(q, L.chunk);
    int rel = at - part[s];
    const int which = rel % parts;  // the blocks of a tile's parts share its rows
    rel /= parts;
    const int h = rel % A.c.n_heads, r0 = rel / A.c.n_heads * R, rows = min(R, q.n * group - r0);
    const float *const from = ws + (int64_t)(at - which) * part_floats(R, D);
    for (int e = which * 256 + threadIdx.x; e < rows * D; e += parts * 256) {
      const int i = e / D, d = e % D;
      float M = kFloor, sum = 0.0f, out = 0.0f;
      for (int p = 0; p < parts; ++p) {
        const float *const f = from + p * part_floats(R, D);
        const float m = f[i], m_new = fmaxf(M, m);
        const float keep = __builtin_amdgcn_exp2f(M - m_new), add = __builtin_amdgcn_exp2f(m - m_new);
        sum = sum * keep + f[R + i] * add;
        out = out * keep + f[2 * R + i * D + d] * add;
        M = m_new;
      }
      const int rr = r0 + i;
      store_value<TYPE>(A.out, ((int64_t)(q.q0 + rr / group) * A.n_q_heads + h * group + rr % group) * D + d,
                        sum == 0.0f ? 0.0f : out / sum);
    }
  }
}

__global__ void k_check_attention(AttendArgs A, int32_t *flag) {
  const int s = blockIdx.x;
  const int q0 = A.cu_q[s], q1 = A.cu_q[s + 1], length = A.ctx_lens[s];
  if (threadIdx.x == 0) {
    if (q0 < 0 || q1 < q0 || q1 > A.n_tokens || (s == 0 && q0 != 0) || (s == A.n_seqs - 1 && q1 != A.n_tokens) ||
        q1 - q0 > A.max_q || length < 0 || length > (A.table_width << A.c.page_shift))
      atomicAdd(&flag[0], 1);
  }
  if (length <= 0 || q1 <= q0) return;
  const int64_t low = A.window ? max((int64_t)0, (int64_t)length - (q1 - q0) - A.window + 1) : 0;
  const int64_t last = min(((int64_t)length - 1) >> A.c.page_shift, A.table_width - 1);
  for (int64_t i = (low >> A.c.page_shift) + threadIdx.x; i <= last; i += blockDim.x) {
    const int32_t id = A.table[s * A.table_width + i];
    if (id < 0 || id >= A.c.n_pages) atomicAdd(&flag[1], 1);
  }
}

// Blocks of the row kernel: four a CU, each with four wavefronts, which holds
// enough loads in flight; at most twice as many parts as its target.
constexpr int kRowBlocks = 1024;

struct Choice {
  int target, least;
};

Choice choose(const AttendArgs &) { return {kRowBlocks, 4}; }

template <int TYPE, int D>
hipError_t attend_as(const AttendArgs &A, float *ws, hipStream_t s) {
  const Choice C = choose(A);
  const size_t lds = 2 * sizeof(int) * A.n_seqs;
  if (lds > 16384) {  // beyond 64 KB with the static part
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_attend_rows<TYPE, D>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  k_attend_rows<TYPE, D><<<kRowBlocks, 256, lds, s>>>(A, C.target, C.least, ws);
  k_join<TYPE, D, kRows><<<kRowBlocks, 256, lds, s>>>(A, C.target, C.least, ws);
  return hipGetLastError();
}

}  // namespace

size_t attention_workspace(const Cache &c, int32_t, int64_t, int32_t) {
  // items of split contexts have at least half a chunk each: at most twice the target
  return 2 * (size_t)kRowBlocks * part_floats(kRows, c.head_dim) * sizeof(float);
}

hipError_t launch_cache_attention(const AttendArgs &A, void *ws, hipStream_t s) {
  float *const w = (float *)ws;
  if (A.type == kF16)
    return A.c.head_dim == 64 ? attend_as<kF16, 64>(A, w, s) : attend_as<kF16, 128>(A, w, s);
  return A.c.head_dim == 64 ? attend_as<kBF16, 64>(A, w, s) : attend_as<kBF16, 128>(A, w, s);
}

hipError_t launch_check_attention(const AttendArgs &A, int32_t *flag, hipStream_t s) {
  k_check_attention<<<A.n_seqs, 64, 0, s>>>(A, flag);
  return hipGetLastError();
}

}  // namespace fs
