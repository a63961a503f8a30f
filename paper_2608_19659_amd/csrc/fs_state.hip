// fs_state.hip -- attention whose past is one matrix a head:
//
//   S_t = l S_(t-1) + k_t v_t^T,   o_t = scale * S_t^T q_t,   l = exp(log_decay)
//
// for packed sequences, the states in a pool.  Two forms of the same sums:
//
// * recurrent, a token at a time with the state in registers, for sequences of
//   few new tokens: bound by the state's bytes, read and written once;
// * in chunks of 64 tokens: with tokens i, j of a chunk and S the state before it,
//     o_i = scale (l^(i+1) S^T q_i + sum_(j <= i) l^(i-j) <q_i, k_j> v_j),
//     S'  = l^n S + sum_j l^(n-1-j) k_j v_j^T,
//   four products on the matrix units.  Long sequences are cut into segments
//   where there are few heads: a pass that makes each segment's own sum, one that
//   adds them up in order, and the outputs from there.
#include <algorithm>

#include "fs_serving.h"

namespace fs {
namespace {

constexpr int kChunk = 64, kThreads = 256;

// Powers of l by exp2 of multiples of its logarithm, which is at least -10^4 here
// so that 0 times it is 0 where l is 0 (log_decay -infinity).  Positive ones count
// as 0; a NaN stays one.
__device__ __forceinline__ float log2_decay(const StateArgs &A, int h) {
  const float x = A.log_decay[h] * 1.44269504f;
  return x > 0.0f ? 0.0f : x < -1e4f ? -1e4f : x;
}
__device__ __forceinline__ float power(float l2, int n) { return __builtin_amdgcn_exp2f(l2 * (float)n); }

struct Sequence {
  int first, count, state;  // state -1: none is read or kept
  bool fresh;               // starts from zeros
};
__device__ __forceinline__ int count_of(const StateArgs &A, int s, int *first) {
  const int a = min(max(A.cu_q[s], 0), A.n_tokens), b = min(max(A.cu_q[s + 1], a), A.n_tokens);
  *first = a;
  return min(b - a, A.max_q);
}
__device__ __forceinline__ Sequence sequence(const StateArgs &A, int s) {
  Sequence q;
  q.count = count_of(A, s, &q.first);
  const int index = A.index[s], held = A.ctx_lens[s];
  q.state = index >= 0 && index < A.n_states ? index : -1;
  q.fresh = q.state < 0 || held <= q.count;
  return q;
}

// ------------------------------------------------------------- token by token --
// A block has COLS columns of a head's state, a thread HELD pieces of four in
// rows ROWS apart.
constexpr int kStepHeads = 8;  // query heads at a time

template <int TYPE, int D, int COLS>
__global__ __launch_bounds__(kThreads) void k_state_step(StateArgs A) {
  constexpr int LANES = COLS / 4, ROWS = kThreads / LANES, HELD = D / ROWS, PARTS = D / COLS, WAVES = kThreads / 64;
  static_assert(HELD >= 1 && LANES <= 64, "a piece a thread at least, a row in a wavefront");
  __shared__ float ks[D], qs[kStepHeads][D], sums[WAVES][kStepHeads][COLS];
  const int part = blockIdx.x % PARTS, h = blockIdx.x / PARTS, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int group = A.n_q_heads / A.n_heads, row = threadIdx.x / LANES, col = threadIdx.x % LANES * 4;
  const Sequence q = sequence(A, blockIdx.y);
  if (q.count < 1 || q.count > A.step_most) return;
  const float l = power(log2_decay(A, h), 1);
  float *const at = q.state < 0 ? nullptr : A.states + ((int64_t)q.state * A.n_heads + h) * D * D + part * COLS + col;
  float4v s[HELD];
#pragma unroll
  for (int i = 0; i < HELD; ++i) s[i] = q.fresh ? float4v{0, 0, 0, 0} : *(const float4v *)(at + (int64_t)(i * ROWS + row) * D);
  for (int t = q.first; t < q.first + q.count; ++t) {
    float4v v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = load_value<TYPE>(A.v, t * A.v_stride + h * D + part * COLS + col + i);
    for (int g0 = 0; g0 < group; g0 += kStepHeads) {
      const int heads = min(kStepHeads, group - g0);
      if (g0 || t > q.first) __syncthreads();
      if (g0 == 0)
        for (int i = threadIdx.x; i < D; i += kThreads) ks[i] = load_value<TYPE>(A.k, t * A.k_stride + h * D + i);
      for (int i = threadIdx.x; i < heads * D; i += kThreads)
        qs[i / D][i % D] = load_value<TYPE>(A.q, t * A.q_stride + ((int64_t)h * group + g0) * D + i);
      __syncthreads();
      if (g0 == 0) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
          const float k = ks[i * ROWS + row];
#pragma unroll
          for (int e = 0; e < 4; ++e) s[i][e] = __builtin_fmaf(k, v[e], l * s[i][e]);
        }
      }
      for (int g = 0; g < heads; ++g) {
        float4v o = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
          const float x = qs[g][i * ROWS + row];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(x, s[i][e], o[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int step = LANES; step < 64; step <<= 1) o[e] += __shfl_xor(o[e], step);
        if (lane < LANES) *(float4v *)&sums[wave][g][col] = o;
      }
      __syncthreads();
      for (int i = threadIdx.x; i < heads * COLS; i += kThreads) {
        const int g = i / COLS, c = i % COLS;
        float o = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) o += sums[w][g][c];
        store_value<TYPE>(A.out, ((int64_t)t * A.n_q_heads + h * group + g0 + g) * D + part * COLS + c, o * A.scale);
      }
    }
  }
  if (q.state < 0) return;
#pragma unroll
  for (int i = 0; i < HELD; ++i) *(float4v *)(at + (int64_t)(i * ROWS + row) * D) = s[i];
}

// ------------------------------------------------------------------ in chunks --
// Segments of `segment` tokens (a multiple of 64), numbered over the sequences;
// sequences of at most step_most tokens have none.
__device__ __forceinline__ int segments(const StateArgs &A, int s) {
  int first;
  const int n = s < A.n_seqs ? count_of(A, s, &first) : 0;
  return n > A.step_most ? (n - 1) / A.segment + 1 : 0;
}
// A sequence of two segments or more has a place in the workspace for each.
__device__ __forceinline__ int places(const StateArgs &A, int s) {
  const int n = segments(A, s);
  return n > 1 ? n : 0;
}
// Places of the sequences before `s` (all of a wavefront's lanes call it).
__device__ __forceinline__ int places_before(const StateArgs &A, int s) {
  int sum = 0;
  for (int i = threadIdx.x & 63; i < s; i += 64) sum += places(A, i);
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  return sum;
}
// (Sequences that overlap, which the call does not allow, may have more segments
// than there are places: those are left out.)
__device__ __forceinline__ bool room_for(const StateArgs &A, int before, int n) { return (int64_t)before + n <= A.n_places; }

__device__ __forceinline__ int sum_upto(int v, int lane) {
  for (int o = 1; o < 64; o <<= 1) {
    const int below = __shfl_up(v, o);
    if (lane >= o) v += below;
  }
  return v;
}
struct Segment {
  int sequence, number, before;  // -1: there is none; its number in the sequence; places before the sequence's
};
__device__ __forceinline__ Segment find_segment(const StateArgs &A, int x) {
  if (A.segment >= A.max_q) return {x, 0, 0};  // a segment a sequence
  const int lane = threadIdx.x & 63;
  int before = 0, taken = 0;
  for (int s0 = 0; s0 < A.n_seqs; s0 += 64) {
    const int n = segments(A, s0 + lane), m = n > 1 ? n : 0, upto = sum_upto(n, lane), took = sum_upto(m, lane);
    const uint64_t in = __ballot(x < before + upto);
    if (in) {
      const int at = __builtin_ctzll(in), first = taken + __shfl(took - m, at);
      if (!room_for(A, first, __shfl(m, at))) break;
      return {s0 + at, x - before - __shfl(upto - n, at), first};
    }
    before += __shfl(upto, 63);
    taken += __shfl(took, 63);
  }
  return {-1, 0, 0};
}

using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using short4v = short __attribute__((ext_vector_type(4)));
using short8v = short __attribute__((ext_vector_type(8)));
using int2v = int __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float4v multiply(short8v a, short8v b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// A binary32 value as the sum of two bfloat16 values: 16 bits of it.  With one
// alone the states, which are binary32, would be off by 2^-9 of a token's share, and
// an output by as much again as its own rounding.
struct Pair {
  short8v hi, lo;
};
__device__ __forceinline__ void split(float x, short &hi, short &lo) {
  const uint16_t h = bf16_bits(x);
  hi = (short)h;
  lo = (short)bf16_bits(x - bf16_value(h));
}

// Tiles of 64 rows in LDS as bfloat16, rows 32 bytes longer than they are, so that
// eight rows' same columns lie on all banks.  binary16 elements are the sums of two
// bfloat16 values (exactly): SPLITS tiles then.
template <int TYPE, int D>
struct Tile {
  static constexpr int SPLITS = TYPE == kF16 ? 2 : 1, PITCH = D + 16, SIZE = kChunk * PITCH;
  static constexpr int PIECES = kChunk * D / 8 / kThreads, PER_ROW = D / 8, STEP = kThreads / PER_ROW;

  // 16 bytes a piece of rows [0, count) from `from` on, zeros behind them.
  __device__ static __forceinline__ void load(const void *from, int64_t stride, int count, bool whole, int4v (&raw)[PIECES]) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int r = threadIdx.x / PER_ROW + i * STEP;
      const uint16_t *const p = (const uint16_t *)from + r * stride + threadIdx.x % PER_ROW * 8;
      raw[i] = r >= count ? int4v{0, 0, 0, 0} : whole ? *(const int4v *)p : load16(p);
    }
  }
  __device__ static __forceinline__ void store(short *tile, const int4v (&raw)[PIECES]) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      short *const to = tile + (threadIdx.x / PER_ROW + i * STEP) * PITCH + threadIdx.x % PER_ROW * 8;
      if constexpr (TYPE == kBF16) {
        *(int4v *)to = raw[i];
      } else {
        Pair p;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          short hi, lo;
          split(f16_value((uint16_t)(raw[i][e >> 1] >> 16 * (e & 1))), hi, lo);
          p.hi[e] = hi;
          p.lo[e] = lo;
        }
        *(short8v *)to = p.hi;
        *(short8v *)(to + SIZE) = p.lo;
      }
    }
  }
  __device__ static __forceinline__ bool finite(const int4v (&raw)[PIECES]) {
    using short2 = uint16_t __attribute__((ext_vector_type(2)));
    short2 most = {0, 0};
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(short2, raw[i][e] & 0x7fff7fff));
    return max(most.x, most.y) < (TYPE == kF16 ? 0x7c00 : 0x7f80);
  }
  // An operand: a lane has row r0 + lane % 16 and columns c + 4 g .. and
  // c + 16 + 4 g .., g = lane / 16: the order in which a product's results lie.
  __device__ static __forceinline__ short8v rows(const short *tile, int r0, int c) {
    const int lane = threadIdx.x & 63;
    const short *const p = tile + (r0 + (lane & 15)) * PITCH + c + (lane >> 4) * 4;
    const short4v a = *(const short4v *)p, b = *(const short4v *)(p + 16);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  // The transpose: a lane has column c + lane % 16 and rows r0 + 4 g .., r0 + 16 + 4 g ..
  __device__ static __forceinline__ short8v columns(const short *tile, int r0, int c) {
    using Place = __attribute__((address_space(3))) short4v;
    const int lane = threadIdx.x & 63, r = lane & 15;
    Place *const p = (Place *)(tile + (r0 + (lane >> 4) * 4 + (r >> 2)) * PITCH + c + (r & 3) * 4);
    const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(p);
    const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Place *)((__attribute__((address_space(3))) short *)p + 16 * PITCH));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// The token of an operand's element e in step t, in the results' order (see rows).
__device__ __forceinline__ constexpr int token(int t, int e, int g) { return t * 32 + (e >> 2) * 16 + 4 * g + (e & 3); }

// Four wavefronts, each with D / 4 of the values' columns.
// SUMS: a segment's own sum to `local`, no outputs.
template <int TYPE, int D, bool SUMS>
struct ChunkShape {
  using T = Tile<TYPE, D>;
  static constexpr int PART = T::SPLITS * T::SIZE;         // a tensor's tiles, in 16-bit words
  static constexpr int PROBS = SUMS ? 0 : 2 * 4 * 2 * 512;  // probabilities, as operands
  static constexpr int BYTES = ((SUMS ? 2 : 3) * PART + PROBS) * 2 + 16;
};

template <int TYPE, int D, bool SUMS>
__global__ __launch_bounds__(kThreads) void k_state_chunk(StateArgs A) {
  using Shape = ChunkShape<TYPE, D, SUMS>;
  using T = Tile<TYPE, D>;
  constexpr int VT = D / 64, KT = D / 16, KS = D / 32, SPLITS = T::SPLITS;  // a wavefront's column tiles; row tiles, steps
  extern __shared__ __attribute__((aligned(16))) short state_lds[];
  short *const lk = state_lds, *const lv = lk + Shape::PART, *const lq = lv + Shape::PART, *const lp = lq + Shape::PART;
  int *const bad = (int *)((char *)state_lds + Shape::BYTES - 16);  // values that are no numbers, of this chunk and the next
  const Segment seg = find_segment(A, blockIdx.x);
  if (seg.sequence < 0) return;
  const Sequence q = sequence(A, seg.sequence);
  if (q.count <= A.step_most) return;
  const int start = seg.number * A.segment, tokens = min(A.segment, q.count - start), h = blockIdx.y;
  const int group = A.n_q_heads / A.n_heads, lane = threadIdx.x & 63, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool last = start + tokens == q.count;
  if (SUMS && last) return;
  const int64_t D2 = (int64_t)D * D;
  float *const local = A.local + ((int64_t)(seg.before + seg.number) * A.n_heads + h) * D2;
  const float l2 = log2_decay(A, h);
  const int dv0 = wave * (D / 4);

  // s[a][b]: rows 16 a + 4 g .. of column dv0 + 16 b + lane % 16
  float4v s[KT][VT] = {};
  const auto place = [&](int a, int b, int e) { return (16 * a + 4 * g + e) * D + dv0 + 16 * b + (lane & 15); };
  if constexpr (!SUMS) {
    const float *from = nullptr;
    // the segments' starts as k_state_join leaves them
    if (seg.number) from = local - (int64_t)A.n_heads * D2;
    else if (!q.fresh) from = last ? A.states + ((int64_t)q.state * A.n_heads + h) * D2
                                   : A.local + ((int64_t)(seg.before + (q.count - 1) / A.segment) * A.n_heads + h) * D2;
    if (from)
#pragma unroll
      for (int a = 0; a < KT; ++a)
#pragma unroll
        for (int b = 0; b < VT; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[a][b][e] = from[place(a, b, e)];
  }

  const int64_t row0 = q.first + start;
  const auto aligned = [](const void *p, int64_t stride) { return (((uintptr_t)p | (uintptr_t)(stride * 2)) & 15) == 0; };
  const bool whole_k = aligned(A.k, A.k_stride), whole_v = aligned(A.v, A.v_stride), whole_q = aligned(A.q, A.q_stride);
  int4v rk[T::PIECES], rv[T::PIECES], rq[T::PIECES];
  const auto ask_kv = [&](int c) {
    const int64_t row = row0 + c;
    T::load((const uint16_t *)A.k + row * A.k_stride + h * D, A.k_stride, tokens - c, whole_k, rk);
    T::load((const uint16_t *)A.v + row * A.v_stride + h * D, A.v_stride, tokens - c, whole_v, rv);
  };
  const auto ask_q = [&](int c, int head) {
    T::load((const uint16_t *)A.q + (row0 + c) * A.q_stride + ((int64_t)h * group + head) * D, A.q_stride, tokens - c, whole_q, rq);
  };
  ask_kv(0);
  if constexpr (!SUMS) ask_q(0, 0);
  if (threadIdx.x < 2) bad[threadIdx.x] = 0;

  // the decay between a token of this wavefront's rows and one before it
  float fade[4][4], seen[4];
  if constexpr (!SUMS) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) fade[j][e] = A.scale * power(l2, max(0, (wave - j) * 16 + (lane & 15) - 4 * g - e));
#pragma unroll
    for (int i = 0; i < 4; ++i) seen[i] = A.scale * power(l2, i * 16 + (lane & 15) + 1);
  }

  for (int c = 0, turn = 0; c < tokens; c += kChunk, turn ^= 1) {
    const int n = min(kChunk, tokens - c);
    __syncthreads();  // the last chunk's tiles are read
    T::store(lk, rk);
    T::store(lv, rv);
    if (!SUMS && !T::finite(rv)) bad[turn] = 1;
    if constexpr (!SUMS) T::store(lq, rq);
    if (c + kChunk < tokens) ask_kv(c + kChunk);
    __syncthreads();
    short8v v[VT][2][SPLITS];
#pragma unroll
    for (int b = 0; b < VT; ++b)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int x = 0; x < SPLITS; ++x) v[b][t][x] = T::columns(lv + x * T::SIZE, t * 32, dv0 + b * 16);
    const bool numbers = SUMS || bad[turn] == 0;
    int none[VT];  // of each column the first token whose value is no number
    if (!numbers) {
      // Tokens before it have a weight of 0 for it, which times it is no number: the
      // products take 0 in its place, and what sees it is made no number behind them.
#pragma unroll
      for (int b = 0; b < VT; ++b) {
        none[b] = kChunk;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if ((v[b][t][0][e] & 0x7f80) == 0x7f80) {
              none[b] = min(none[b], token(t, e, g));
#pragma unroll
              for (int x = 0; x < SPLITS; ++x) v[b][t][x][e] = 0;
            }
        for (int o = 16; o < 64; o <<= 1) none[b] = min(none[b], __shfl_xor(none[b], o));
      }
    }
    if constexpr (!SUMS) {
      Pair past[VT][KS];  // the state as an operand: its results' order is the operands'
#pragma unroll
      for (int b = 0; b < VT; ++b)
#pragma unroll
        for (int t = 0; t < KS; ++t)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            short hi, lo;
            split(s[2 * t + (e >> 2)][b][e & 3], hi, lo);
            past[b][t].hi[e] = hi;
            past[b][t].lo[e] = lo;
          }
      for (int head = 0; head < group; ++head) {
        if (head) {
          __syncthreads();
          T::store(lq, rq);
          __syncthreads();
        }
        if (head + 1 < group) ask_q(c, head + 1);
        else if (c + kChunk < tokens) ask_q(c + kChunk, 0);
        // this wavefront's 16 rows of <q, k>, decayed, to LDS as operands
        {
          short8v mine[KS][SPLITS];
#pragma unroll
          for (int t = 0; t < KS; ++t)
#pragma unroll
            for (int x = 0; x < SPLITS; ++x) mine[t][x] = T::rows(lq + x * T::SIZE, wave * 16, t * 32);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            Pair p = {};
            if (2 * t <= wave) {
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                const int j = 2 * t + half;
                if (j > wave) continue;
                float4v sum = {0, 0, 0, 0};
#pragma unroll
                for (int d = 0; d < KS; ++d) {
                  const short8v k = T::rows(lk, j * 16, d * 32);
                  sum = multiply(k, mine[d][0], sum);
                  if constexpr (SPLITS == 2) {
                    sum = multiply(k, mine[d][1], sum);
                    sum = multiply(T::rows(lk + T::SIZE, j * 16, d * 32), mine[d][0], sum);
                  }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  // later tokens are left out, whatever they are
                  const float x = j == wave && 4 * g + e > (lane & 15) ? 0.0f : sum[e] * fade[j][e];
                  short hi, lo;
                  split(x, hi, lo);
                  p.hi[half * 4 + e] = hi;
                  p.lo[half * 4 + e] = lo;
                }
              }
              *(short8v *)(lp + ((wave * 2 + t) * 64 + lane) * 8) = p.hi;
              *(short8v *)(lp + 4096 + ((wave * 2 + t) * 64 + lane) * 8) = p.lo;
            }
          }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i * 16 >= n) break;
          float4v o[VT] = {};
#pragma unroll
          for (int t = 0; t < KS; ++t) {
            const short8v x = T::rows(lq, i * 16, t * 32);
#pragma unroll
            for (int b = 0; b < VT; ++b) {
              o[b] = multiply(past[b][t].hi, x, o[b]);
              o[b] = multiply(past[b][t].lo, x, o[b]);
            }
            if constexpr (SPLITS == 2) {
              const short8v y = T::rows(lq + T::SIZE, i * 16, t * 32);
#pragma unroll
              for (int b = 0; b < VT; ++b) o[b] = multiply(past[b][t].hi, y, o[b]);
            }
          }
#pragma unroll
          for (int b = 0; b < VT; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[b][e] *= seen[i];
#pragma unroll
          for (int t = 0; t <= i / 2; ++t) {
            const short8v hi = *(const short8v *)(lp + ((i * 2 + t) * 64 + lane) * 8);
            const short8v lo = *(const short8v *)(lp + 4096 + ((i * 2 + t) * 64 + lane) * 8);
#pragma unroll
            for (int b = 0; b < VT; ++b) {
              o[b] = multiply(v[b][t][0], hi, o[b]);
              o[b] = multiply(v[b][t][0], lo, o[b]);
              if constexpr (SPLITS == 2) o[b] = multiply(v[b][t][1], hi, o[b]);
            }
          }
          if (!numbers) {
#pragma unroll
            for (int b = 0; b < VT; ++b)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (i * 16 + (lane & 15) >= __shfl(none[b], 4 * g + e)) o[b][e] = __builtin_nanf("");
          }
          const int row = c + i * 16 + (lane & 15);
          if (row < tokens) {
#pragma unroll
            for (int b = 0; b < VT; ++b) {
              uint16_t bits[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) bits[e] = bits16<TYPE>(o[b][e]);
              __builtin_memcpy((uint16_t *)A.out + ((row0 + row) * A.n_q_heads + h * group + head) * D + dv0 + b * 16 + 4 * g, bits, 8);
            }
          }
        }
      }
      if (threadIdx.x == 0) bad[turn ^ 1] = 0;
      if (last && q.state < 0 && c + kChunk >= tokens) return;
    }
    // the state after the chunk
    const float kept = power(l2, n);
    Pair fading[VT][2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float w = power(l2, max(0, n - 1 - token(t, e, g)));
#pragma unroll
        for (int b = 0; b < VT; ++b) {
          float x = bf16_value((uint16_t)v[b][t][0][e]);
          if constexpr (SPLITS == 2) x += bf16_value((uint16_t)v[b][t][1][e]);
          if (!numbers && token(t, e, g) == none[b]) x = __builtin_nanf("");
          short hi, lo;
          split(x * w, hi, lo);
          fading[b][t].hi[e] = hi;
          fading[b][t].lo[e] = lo;
        }
      }
#pragma unroll
    for (int a = 0; a < KT; ++a) {
#pragma unroll
      for (int b = 0; b < VT; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[a][b][e] *= kept;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const short8v k = T::columns(lk, t * 32, a * 16);
#pragma unroll
        for (int b = 0; b < VT; ++b) {
          s[a][b] = multiply(k, fading[b][t].hi, s[a][b]);
          s[a][b] = multiply(k, fading[b][t].lo, s[a][b]);
        }
        if constexpr (SPLITS == 2) {
          const short8v y = T::columns(lk + T::SIZE, t * 32, a * 16);
#pragma unroll
          for (int b = 0; b < VT; ++b) s[a][b] = multiply(y, fading[b][t].hi, s[a][b]);
        }
      }
    }
  }
  float *to = nullptr;
  if constexpr (SUMS) to = local;
  else if (last && q.state >= 0) to = A.states + ((int64_t)q.state * A.n_heads + h) * D2;
  if (to)
#pragma unroll
    for (int a = 0; a < KT; ++a)
#pragma unroll
      for (int b = 0; b < VT; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) to[place(a, b, e)] = s[a][b][e];
}

// A sequence's segments in order: local[j] becomes the state after segment j, and
// the place of the last, which made no sum, takes the state that the sequence
// starts from (its own may be written by the last segment while the first reads).
template <int D>
__global__ __launch_bounds__(kThreads) void k_state_join(StateArgs A) {
  constexpr int PIECES = D * D / 4 / kThreads;
  const int piece = blockIdx.x % PIECES, h = blockIdx.x / PIECES, n = segments(A, blockIdx.y);
  if (n < 2) return;
  const Sequence q = sequence(A, blockIdx.y);
  const int64_t D2 = (int64_t)D * D, step = A.n_heads * D2, at = (piece * kThreads + threadIdx.x) * 4;
  const int before = places_before(A, blockIdx.y);
  if (!room_for(A, before, n)) return;
  float *p = A.local + ((int64_t)before * A.n_heads + h) * D2 + at;
  const float kept = power(log2_decay(A, h), A.segment);
  float4v s = {0, 0, 0, 0};
  if (!q.fresh) s = *(const float4v *)(A.states + ((int64_t)q.state * A.n_heads + h) * D2 + at);
  *(float4v *)(p + (n - 1) * step) = s;
  for (int j = 0; j + 1 < n; ++j, p += step) {
    const float4v own = *(const float4v *)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = __builtin_fmaf(kept, s[e], own[e]);
    *(float4v *)p = s;
  }
}

__global__ void k_check_state(StateArgs A, int32_t *flag) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < A.n_heads && !(A.log_decay[i] <= 0.0f)) atomicAdd(&flag[1], 1);
  if (i >= A.n_seqs) return;
  const int a = A.cu_q[i], b = A.cu_q[i + 1], at = A.index[i];
  bool wrong = (i == 0 && a != 0) || a < 0 || b < a || b > A.n_tokens || b - a > A.max_q || A.ctx_lens[i] < 0 || at >= A.n_states;
  if (at >= 0 && b > a)
    for (int j = 0; j < i; ++j) wrong |= A.index[j] == at && A.cu_q[j + 1] > A.cu_q[j];
  if (wrong) atomicAdd(&flag[0], 1);
}

// Sequences of up to this many new tokens go token by token.
constexpr int kStepMost = 8;

// Tokens of a segment: one for each sequence where the heads fill the CUs, else so
// many that about 512 segments and heads come out.
int segment_tokens(int64_t n_tokens, int64_t n_heads) {
  const int64_t L = (n_tokens * n_heads / 512 + 63) / 64 * 64;
  return (int)std::max<int64_t>(256, std::min<int64_t>(L, 1 << 30));
}
int64_t segments_at_most(int64_t n_tokens, int64_t n_seqs, int64_t n_heads) {
  return n_tokens / segment_tokens(n_tokens, n_heads) + n_seqs;
}
// Of sequences of more than a segment's L tokens: n of them have at most n / L + 1,
// less than 2 n / L.
int64_t places_at_most(int64_t n_tokens, int64_t n_heads) {
  const int64_t L = segment_tokens(n_tokens, n_heads);
  return n_tokens > L ? 2 * n_tokens / L : 0;
}

template <class K>
hipError_t launch_chunks(K kernel, int bytes, dim3 grid, const StateArgs &A, hipStream_t s) {
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != hipSuccess) return e;
  kernel<<<grid, kThreads, bytes, s>>>(A);
  return hipGetLastError();
}

template <int TYPE, int D, int COLS>
hipError_t steps_as(const StateArgs &A, hipStream_t s) {
  k_state_step<TYPE, D, COLS><<<dim3(A.n_heads * (D / COLS), A.n_seqs), kThreads, 0, s>>>(A);
  return hipGetLastError();
}

template <int TYPE, int D>
hipError_t state_of(StateArgs A, hipStream_t s) {
  hipError_t e = hipSuccess;
  A.step_most = A.max_q > kStepMost && A.n_seqs == 1 ? 0 : kStepMost;
  if (A.step_most) {
    const int64_t heads = (int64_t)A.n_seqs * A.n_heads;
    if (heads >= 512) e = steps_as<TYPE, D, D>(A, s);
    else if (heads >= 128) e = steps_as<TYPE, D, 32>(A, s);
    else e = steps_as<TYPE, D, 16>(A, s);
    if (e != hipSuccess || A.max_q <= kStepMost) return e;
  }
  A.segment = segment_tokens(A.n_tokens, A.n_heads);
  if (A.segment >= A.max_q)
    return launch_chunks(k_state_chunk<TYPE, D, false>, ChunkShape<TYPE, D, false>::BYTES, dim3(A.n_seqs, A.n_heads), A, s);
  A.n_places = (int32_t)places_at_most(A.n_tokens, A.n_heads);
  const dim3 grid((unsigned)segments_at_most(A.n_tokens, A.n_seqs, A.n_heads), A.n_heads);
  e = launch_chunks(k_state_chunk<TYPE, D, true>, ChunkShape<TYPE, D, true>::BYTES, grid, A, s);
  if (e != hipSuccess) return e;
  k_state_join<D><<<dim3(A.n_heads * (D * D / 4 / kThreads), A.n_seqs), kThreads, 0, s>>>(A);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_chunks(k_state_chunk<TYPE, D, false>, ChunkShape<TYPE, D, false>::BYTES, grid, A, s);
}

}  // namespace

size_t state_workspace(int32_t n_heads, int32_t head_dim, int64_t n_tokens) {
  return (size_t)(places_at_most(n_tokens, n_heads) * n_heads * head_dim * head_dim) * 4;
}

hipError_t launch_check_state(const StateArgs &A, int32_t *flag, hipStream_t s) {
  k_check_state<<<(std::max(A.n_seqs, A.n_heads) - 1) / 256 + 1, 256, 0, s>>>(A, flag);
  return hipGetLastError();
}

hipError_t launch_state_attention(const StateArgs &A, hipStream_t s) {
  if (A.head_dim == 64) return A.type == kF16 ? state_of<kF16, 64>(A, s) : state_of<kBF16, 64>(A, s);
  return A.type == kF16 ? state_of<kF16, 128>(A, s) : state_of<kBF16, 128>(A, s);
}

}  // namespace fs
