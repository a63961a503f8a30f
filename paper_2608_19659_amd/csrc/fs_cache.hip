// fs_cache.hip -- the paged 8-bit key/value cache: appending a step's tokens
// with the position rotation applied on the way, and reading values back.
#include <algorithm>

#include "fs_serving.h"

namespace fs {
namespace {

__device__ int32_t g_flag[2];  // FS_VALIDATE=1: what the checks counted

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ int64_t n_slots(const Cache &c) { return (int64_t)c.n_pages << c.page_shift; }

// The code of a value under the inverse of its scale.
__device__ __forceinline__ int code_of(float x, float inverse) {
  return (int)fminf(fmaxf(rintf(x * inverse), -127.0f), 127.0f);
}

__device__ __forceinline__ int position_of(const AppendArgs &A, int t) {
  return A.half ? min(max(A.positions[t], 0), A.n_positions - 1) : 0;
}

// The codes of eight values, packed.
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float inverse) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i >> 2] |= (uint32_t)(code_of(v[i], inverse) & 0xff) << (8 * (i & 3));
  return {w[0], w[1]};
}

// Sixteen elements of a head's row, as two neighbouring eights at d[0], d[1].
// A rotation of 16 m elements has its partners in one piece: pieces 0 .. m - 1
// are eights of the first half with those of the second, later ones neighbours.
struct Piece {
  float v[2][8];
  int d[2];

  __device__ __forceinline__ void place(int c, int half) {
    const bool pair = c * 8 < half;
    d[0] = pair ? c * 8 : c * 16;
    d[1] = pair ? half + c * 8 : c * 16 + 8;
  }
};

// x' = x cos -+ partner sin, each product and sum rounded.  EVEN: the rotated
// part is a multiple of 16 elements.
template <int TYPE, bool EVEN>
__device__ __forceinline__ void load_rotated(const AppendArgs &A, const void *x, int64_t row, bool whole, int c, int position,
                                             Piece &p) {
  const int64_t at = (int64_t)position * A.half;
  if constexpr (EVEN) {
    p.place(c, A.half);
    load8<TYPE>(x, row + p.d[0], whole, p.v[0]);
    load8<TYPE>(x, row + p.d[1], whole, p.v[1]);
    if (A.half == 0) return;
    // pieces that are not rotated: by an angle of 0, with the first one's loads
    const bool turned = c * 8 < A.half;
    float co[8], si[8];
    __builtin_memcpy(co, A.cosines + at + (turned ? c * 8 : 0), 32);
    __builtin_memcpy(si, A.sines + at + (turned ? c * 8 : 0), 32);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = p.v[0][i], b = p.v[1][i];
      const float x0 = a * co[i] - b * si[i], x1 = b * co[i] + a * si[i];
      p.v[0][i] = turned ? x0 : a;
      p.v[1][i] = turned ? x1 : b;
    }
  } else {
    p.place(c, 0);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int d = c * 16 + i;
      float v = load_value<TYPE>(x, row + d);
      if (d < 2 * A.half) {
        const bool low = d < A.half;
        const int k = low ? d : d - A.half;
        const float w = load_value<TYPE>(x, row + (low ? d + A.half : k)), co = A.cosines[at + k], si = A.sines[at + k];
        v = low ? v * co - w * si : v * co + w * si;
      }
      p.v[i >> 3][i & 7] = v;
    }
  }
}

template <int TYPE>
bool starts_whole(const void *x, int64_t stride) {  // rows on multiples of 16 bytes
  return (((uintptr_t)x | (uintptr_t)(stride * (TYPE == kF32 ? 4 : 2))) & 15) == 0;
}

// One page's keys (or values) of one head: the new tokens in registers, their
// largest magnitude, the page's new scale, then the codes.  The codes held are
// read and written only where the scale grows, but for the 16 tokens of values
// around a new one: those share a store.
template <int TYPE, int D, bool VALUES, bool EVEN>
__device__ void append_page(const AppendArgs &A, int t, int slot, int head, bool whole, int8_t *lds, uint32_t *most) {
  constexpr int PIECES = D / 16, HELD = 64 * PIECES / 256, ROW = 68;  // LDS row of an element's codes: 64 tokens, padded
  const Cache &c = A.c;
  const int PS = 1 << c.page_shift, lane = threadIdx.x & 63;
  const int first = slot & (PS - 1);
  // the new tokens of this page: those that follow in the slots that follow
  const bool next = lane < PS - first && t + lane < A.n_tokens && A.slots[min(t + lane, A.n_tokens - 1)] == slot + lane;
  const uint64_t mask = __ballot(next);
  const int n = mask == ~0ull ? 64 : __ffsll((unsigned long long)~mask) - 1;
  const int64_t block = (int64_t)(slot >> c.page_shift) * c.n_heads + head;
  float *const scale = (VALUES ? c.v_scale : c.k_scale) + block;
  int8_t *const codes = (VALUES ? c.v : c.k) + block * PS * D;
  const float old = first ? *scale : 0.0f;
  const void *const x = VALUES ? A.v : A.k;
  const int64_t stride = VALUES ? A.v_stride : A.k_stride;
  if (threadIdx.x == 0) *most = 0;
  __syncthreads();
  Piece p[HELD];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    // beyond the new tokens the last again: with no condition all loads are under way together
    const int e = threadIdx.x + 256 * i, j = min(e / PIECES, n - 1), piece = e % PIECES;
    const int64_t row = (int64_t)(t + j) * stride + head * D;
    if constexpr (VALUES) {
      p[i].place(piece, 0);
      load8<TYPE>(x, row + p[i].d[0], whole, p[i].v[0]);
      load8<TYPE>(x, row + p[i].d[1], whole, p[i].v[1]);
    } else {
      load_rotated<TYPE, EVEN>(A, x, row, whole, piece, position_of(A, t + j), p[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < HELD; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) m = max(m, max(magnitude(p[i].v[0][k]), magnitude(p[i].v[1][k])));
  for (int o = 32; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
  if (lane == 0) atomicMax(most, m);
  __syncthreads();
  const float a = __uint_as_float(*most), made = a < kTiny ? 0.0f : a / 127.0f;
  float now = old >= made || old != old ? old : made;  // a NaN on either side stays
  now += now - now;                                    // and an infinity, which no code can stand beside, becomes one
  const bool grew = first && !(now == old);
  const float inverse = now > 0.0f ? 1.0f / now : 0.0f, ratio = now > 0.0f ? old / now : 0.0f;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int j = (threadIdx.x + 256 * i) / PIECES;
    if (j >= n) continue;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint2 w = codes8(p[i].v[k], inverse);
      if constexpr (VALUES) {
#pragma unroll
        for (int b = 0; b < 8; ++b) lds[(p[i].d[k] + b) * ROW + first + j] = (int8_t)((b < 4 ? w.x : w.y) >> (8 * (b & 3)));
      } else {
        *(uint2 *)(codes + (first + j) * D + p[i].d[k]) = w;
      }
    }
  }
  if constexpr (VALUES) {  // a thread owns 16 tokens of one element
    __syncthreads();
    const int g0 = grew ? 0 : first >> 4, g1 = (first + n - 1) >> 4, ng = g1 - g0 + 1;
    for (int e = threadIdx.x; e < D * ng; e += 256) {
      const int d = ng == 4 ? e >> 2 : e / ng, g = g0 + e - d * ng;
      int4v *const to = (int4v *)(codes + d * PS + g * 16);
      const int *const made_row = (const int *)(lds + d * ROW + g * 16);
      int4v row = {made_row[0], made_row[1], made_row[2], made_row[3]};
      if (g * 16 < first || g * 16 + 16 > first + n) {
        const int4v held = *to;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = g * 16 + i, shift = 8 * (i & 3);
          if (at >= first && at < first + n) continue;
          int code = (int)(int8_t)(held[i >> 2] >> shift);
          if (grew && at < first) code = (int)rintf((float)code * ratio);
          row[i >> 2] = (row[i >> 2] & ~(0xff << shift)) | ((code & 0xff) << shift);
        }
      }
      *to = row;
    }
  } else if (grew) {
    for (int e = threadIdx.x; e < first * (D / 4); e += 256) {
      const uint32_t held = ((const uint32_t *)codes)[e];
      uint32_t w = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) w |= (uint32_t)((int)rintf((float)(int8_t)(held >> 8 * i) * ratio) & 0xff) << 8 * i;
      ((uint32_t *)codes)[e] = w;
    }
  }
  if (threadIdx.x == 0) *scale = now;
  __syncthreads();
}

// blockIdx.x, z: a run of `span` tokens; blockIdx.y: the keys and the values of
// each cache head, then blocks of query heads.
// WHOLE: all rows start on multiples of 16 bytes.
template <int TYPE, int D, bool EVEN, bool WHOLE>
__global__ __launch_bounds__(256) void k_append(AppendArgs A, int span) {
  __shared__ __attribute__((aligned(16))) int8_t lds[D * 68];
  __shared__ uint32_t most;
  constexpr int PIECES = D / 16;
  const int PS = 1 << A.c.page_shift;
  // A prompt's pages start every gridDim.z runs; those runs, which have the work,
  // come first, and one after the other they go round all the XCDs and CUs (in
  // the order of tokens a few of the CUs had them all: 33 us instead of 17 for
  // 8192 tokens of 8 heads).
  const int at_run = blockIdx.x * gridDim.z + blockIdx.z;
  if (at_run > (A.n_tokens - 1) / span) return;
  const int t0 = at_run * span, t1 = min(t0 + span, A.n_tokens);
  const int first_q = 2 * A.c.n_heads, part = blockIdx.y, lane = threadIdx.x & 63;
  if (part < first_q) {
    // the run's tokens that are the first new ones of their pages; the others
    // are done with those
    int slot = -1;
    bool leads = false;
    if (t0 + lane < t1) {
      slot = A.slots[t0 + lane];
      const int before = t0 + lane > 0 ? A.slots[t0 + lane - 1] : -1;
      leads = slot >= 0 && slot < n_slots(A.c) && (!(slot & (PS - 1)) || before != slot - 1);
    }
    for (uint64_t left = __ballot(leads); left; left &= left - 1) {
      const int at = __ffsll((unsigned long long)left) - 1, s = __shfl(slot, at);
      if (part & 1) append_page<TYPE, D, true, EVEN>(A, t0 + at, s, part >> 1, WHOLE, lds, &most);
      else append_page<TYPE, D, false, EVEN>(A, t0 + at, s, part >> 1, WHOLE, lds, &most);
    }
    return;
  }
  const int pieces = A.n_q_heads * PIECES, step = (gridDim.y - first_q) * 256;
  const int all = (t1 - t0) * pieces;
  for (int e0 = (part - first_q) * 256 + threadIdx.x; e0 < all; e0 += 2 * step) {
    Piece p[2];  // two under way at a time (at the end the last again)
    int64_t to[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int e = min(e0 + k * step, all - 1), i = e / pieces, t = t0 + i, head = (e - i * pieces) / PIECES;
      load_rotated<TYPE, EVEN>(A, A.q, (int64_t)t * A.q_stride + head * D, WHOLE, e % PIECES, position_of(A, t), p[k]);
      to[k] = ((int64_t)t * A.n_q_heads + head) * D;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (e0 + k * step >= all) break;
      store8<TYPE>(A.q_out, to[k] + p[k].d[0], p[k].v[0]);
      store8<TYPE>(A.q_out, to[k] + p[k].d[1], p[k].v[1]);
    }
  }
}

// A block reads 16 tokens of one head: half of its wavefronts keys, four
// neighbouring elements a lane; half values, an element a lane, whose 16
// tokens mostly lie in one or two words of 16.
template <int TYPE, int D>
__global__ __launch_bounds__(256) void k_read(ReadArgs A) {
  __shared__ __attribute__((aligned(16))) int8_t lds[D * 36];
  const Cache &c = A.c;
  const int PS = 1 << c.page_shift, lane = threadIdx.x & 63;
  const int t0 = blockIdx.x * 16, head = blockIdx.y, n = min(16, A.n_tokens - t0);
  const int mine = A.slots[t0 + min(lane & 15, n - 1)];
  const auto block_of = [&](int slot) { return (int64_t)(slot >> c.page_shift) * c.n_heads + head; };
  const auto inside = [&](int slot) { return slot >= 0 && slot < n_slots(c); };
  if (threadIdx.x < 128) {
    if (!A.k_out) return;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      const int e = threadIdx.x + 128 * k, i = e / (D / 4), d = e % (D / 4) * 4;
      const int slot = __shfl(mine, i);
      float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      if (inside(slot)) {
        const int64_t block = block_of(slot);
        const uint32_t w = *(const uint32_t *)(c.k + (block * PS + (slot & (PS - 1))) * D + d);
        const float scale = c.k_scale[block];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)(int8_t)(w >> 8 * j) * scale;
      }
      if (i >= n) continue;
      const int64_t to = ((int64_t)(t0 + i) * c.n_heads + head) * D + d;
      if constexpr (TYPE == kF32) {
        __builtin_memcpy((float *)A.k_out + to, v, 16);
      } else {
        const uint2 w = {bits16<TYPE>(v[0]) | (uint32_t)bits16<TYPE>(v[1]) << 16, bits16<TYPE>(v[2]) | (uint32_t)bits16<TYPE>(v[3]) << 16};
        __builtin_memcpy((uint16_t *)A.k_out + to, &w, 8);
      }
    }
    return;
  }
  if (!A.v_out) return;
  const int a = __shfl(mine, 0) >> 4, b = __shfl(mine, n - 1) >> 4;
  const bool two = __all(inside(mine) && (mine >> 4 == a || mine >> 4 == b));
  const float scale_of = c.v_scale[two ? block_of(mine) : 0];
  const int d = threadIdx.x - 128;
  if (d >= D) return;
  const int64_t to = ((int64_t)t0 * c.n_heads + head) * D + d, next = (int64_t)c.n_heads * D;
  if (two) {
    const auto word = [&](int g) { return *(const int4v *)(c.v + (block_of(g << 4) * D + d) * PS + ((g << 4) & (PS - 1))); };
    int *const row = (int *)(lds + d * 36);
    const int4v wa = word(a), wb = word(b);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      row[j] = wa[j];
      row[4 + j] = wb[j];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int slot = __builtin_amdgcn_readlane(mine, i);
      const float scale = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(scale_of), i));
      const float v = (float)lds[d * 36 + (slot >> 4 == a ? 0 : 16) + (slot & 15)] * scale;
      if (i < n) store_value<TYPE>(A.v_out, to + i * next, v);
    }
  } else {
    for (int i = 0; i < n; ++i) {
      const int slot = __builtin_amdgcn_readlane(mine, i);
      float v = 0.0f;
      if (inside(slot)) {
        const int64_t block = block_of(slot);
        v = (float)c.v[(block * D + d) * PS + (slot & (PS - 1))] * c.v_scale[block];
      }
      store_value<TYPE>(A.v_out, to + i * next, v);
    }
  }
}

__global__ void k_clear(int32_t *flag) {
  if (threadIdx.x < 2) flag[threadIdx.x] = 0;
}

__global__ void k_check_slots(Cache c, const int32_t *slots, const int32_t *positions, int32_t n_positions, int32_t n,
                              int appending, int32_t *flag) {
  const int64_t t = blockIdx.x * (int64_t)256 + threadIdx.x;
  if (t >= n) return;
  const int slot = slots[t];
  if (slot >= n_slots(c) || (slot < 0 && !appending)) atomicAdd(&flag[0], 1);
  if (positions && (positions[t] < 0 || positions[t] >= n_positions)) atomicAdd(&flag[1], 1);
}

}  // namespace

hipError_t flag_address(int32_t **flag) { return hipGetSymbolAddress((void **)flag, HIP_SYMBOL(g_flag)); }

hipError_t launch_clear_flag(int32_t *flag, hipStream_t s) {
  k_clear<<<1, 64, 0, s>>>(flag);
  return hipGetLastError();
}

hipError_t launch_check_slots(const Cache &c, const int32_t *slots, const int32_t *positions, int32_t n_positions,
                              int32_t n_tokens, int appending, int32_t *flag, hipStream_t s) {
  k_check_slots<<<(n_tokens - 1) / 256 + 1, 256, 0, s>>>(c, slots, positions, n_positions, n_tokens, appending, flag);
  return hipGetLastError();
}

template <int TYPE, int D, bool EVEN>
static hipError_t append_as(const AppendArgs &A, hipStream_t s) {
  // few tokens a block while that is few blocks: each may be a page of its own
  const int span = A.n_tokens <= 512 ? 1 : A.n_tokens <= 2048 ? 4 : 16;
  const int q_blocks = A.q ? std::min(16, (span * A.n_q_heads * (D / 16) + 511) / 512) : 0;
  const int runs = (A.n_tokens - 1) / span + 1;
  const int fold = std::max({(1 << A.c.page_shift) / span, 1, (int)((runs - 1) / kMostBlocks) + 1});
  const dim3 grid((runs + fold - 1) / fold, 2 * A.c.n_heads + q_blocks, fold);
  const bool whole = starts_whole<TYPE>(A.k, A.k_stride) && starts_whole<TYPE>(A.v, A.v_stride) &&
                     (!A.q || starts_whole<TYPE>(A.q, A.q_stride));
  if (whole) k_append<TYPE, D, EVEN, true><<<grid, 256, 0, s>>>(A, span);
  else k_append<TYPE, D, EVEN, false><<<grid, 256, 0, s>>>(A, span);
  return hipGetLastError();
}

template <int TYPE>
static hipError_t append_of(const AppendArgs &A, hipStream_t s) {
  const bool even = A.half % 8 == 0;
  if (A.c.head_dim == 64) return even ? append_as<TYPE, 64, true>(A, s) : append_as<TYPE, 64, false>(A, s);
  return even ? append_as<TYPE, 128, true>(A, s) : append_as<TYPE, 128, false>(A, s);
}

hipError_t launch_cache_append(const AppendArgs &A, hipStream_t s) {
  return A.type == kF32 ? append_of<kF32>(A, s) : A.type == kF16 ? append_of<kF16>(A, s) : append_of<kBF16>(A, s);
}

template <int TYPE>
static hipError_t read_of(const ReadArgs &A, hipStream_t s) {
  const int64_t element = TYPE == kF32 ? 4 : 2, token = A.c.n_heads * (int64_t)A.c.head_dim * element;
  for (int64_t t = 0; t < A.n_tokens; t += kMostBlocks * 16) {
    ReadArgs part = A;
    part.slots = A.slots + t;
    part.n_tokens = (int32_t)std::min(kMostBlocks * 16, A.n_tokens - t);
    if (A.k_out) part.k_out = (uint8_t *)A.k_out + t * token;
    if (A.v_out) part.v_out = (uint8_t *)A.v_out + t * token;
    const dim3 grid((part.n_tokens + 15) / 16, A.c.n_heads);
    if (A.c.head_dim == 64) k_read<TYPE, 64><<<grid, 256, 0, s>>>(part);
    else k_read<TYPE, 128><<<grid, 256, 0, s>>>(part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_cache_read(const ReadArgs &A, hipStream_t s) {
  return A.type == kF32 ? read_of<kF32>(A, s) : A.type == kF16 ? read_of<kF16>(A, s) : read_of<kBF16>(A, s);
}

}  // namespace fs
