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
#include <cmath>

#include "fs_serving.h"

namespace fs {
namespace {

constexpr int kChunk = 64, kThreads = 256;  // kThreads: of a block that goes token by token, or joins

// Powers of l up to 127 by exp2 of multiples of its logarithm, which is at least -10^4
// here so that 0 times it is 0 where l is 0 (log_decay -infinity).  Positive ones count
// as 0; a NaN stays one.  The logarithm in two parts, the first of 17 bits, whose
// multiples are exact, the second as the factor 1 + its multiple: a far token's power
// is off by two steps like a near one's (a logarithm of 24 bits, times 100, would be off
// by 2^-17 of the power).
struct Rate {
  float upper, lower;
};
__device__ __forceinline__ Rate log2_decay(const StateArgs &A, int h) {
  const double exact = (double)A.log_decay[h] * 1.4426950408889634, x = exact > 0.0 ? 0.0 : exact < -1e4 ? -1e4 : exact;
  const float upper = __uint_as_float((__float_as_uint((float)x) + 0x40) & ~0x7fu);
  return {upper, (float)((x - (double)upper) * 0.6931471805599453)};
}
__device__ __forceinline__ float power(Rate l, float n) {
  const float p = __builtin_amdgcn_exp2f(l.upper * n);
  return __builtin_fmaf(p, l.lower * n, p);
}

// The same to the last bit: what a state is multiplied by once for many tokens.
__device__ __forceinline__ float exact_power(const StateArgs &A, int h, int n) {
  const float x = A.log_decay[h];
  return (float)exp((x > 0.0f ? 0.0 : (double)x) * n);
}

struct Sequence {
  int first, count, state;  // state -1: none is read or kept
  bool fresh;               // starts from zeros
};
__device__ __forceinline__ int count_of(const StateArgs &A, int s, int *first) {
  const int a = min(max(A.cu_q[s], 0), A.n_tokens), b = min(max(A.cu_q[s + 1], a), A.n_tokens);
  *first = a;
  return min(b - a, A.max_q);
}
__device__ __forceinline__ Sequence sequence_of(const StateArgs &A, int first, int count, int index, int held) {
  Sequence q;
  q.first = first;
  q.count = count;
  q.state = index >= 0 && index < A.n_states ? index : -1;
  q.fresh = q.state < 0 || held <= q.count;
  return q;
}
__device__ __forceinline__ Sequence sequence(const StateArgs &A, int s) {
  int first;
  const int count = count_of(A, s, &first);
  return sequence_of(A, first, count, A.index[s], A.ctx_lens[s]);
}

// ------------------------------------------------------------------- segments --
// Segments of `segment` tokens (a multiple of 64), numbered over the sequences;
// sequences of at most step_most tokens have none.
__device__ __forceinline__ int segments_in(const StateArgs &A, int count) { return count > A.step_most ? (count - 1) / A.segment + 1 : 0; }
__device__ __forceinline__ int segments(const StateArgs &A, int s) {
  int first;
  return s < A.n_seqs ? segments_in(A, count_of(A, s, &first)) : 0;
}
// A sequence of two segments or more has a place in the workspace for each.
__device__ __forceinline__ int places(const StateArgs &A, int s) {
  const int n = segments(A, s);
  return n > 1 ? n : 0;
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
  int number, before;  // its number in the sequence; -1: there is none; places before the sequence's
  Sequence sequence;
};
__device__ __forceinline__ Segment find_segment(const StateArgs &A, int x) {
  if (A.segment >= A.max_q) return {0, 0, sequence(A, x)};  // a segment a sequence
  const int lane = threadIdx.x & 63;
  int before = 0, taken = 0;
  for (int s0 = 0; s0 < A.n_seqs; s0 += 64) {
    const int s = min(s0 + lane, A.n_seqs - 1);
    int first;  // all loads at once: the block can do nothing without them
    const int count = count_of(A, s, &first), index = A.index[s], held = A.ctx_lens[s];
    const int n = s0 + lane < A.n_seqs ? segments_in(A, count) : 0, m = n > 1 ? n : 0;
    const int upto = sum_upto(n, lane), took = sum_upto(m, lane);
    const uint64_t in = __ballot(x < before + upto);
    if (in) {
      const int at = __builtin_ctzll(in), place = taken + __shfl(took - m, at);
      if (!room_for(A, place, __shfl(m, at))) break;
      return {x - before - __shfl(upto - n, at), place,
              sequence_of(A, __shfl(first, at), __shfl(count, at), __shfl(index, at), __shfl(held, at))};
    }
    before += __shfl(upto, 63);
    taken += __shfl(took, 63);
  }
  return {-1, 0, {}};
}

// Sequence by sequence of those in segments: the segments in order.  local[j] becomes
// the state after segment j, and the place of the last, which made no sum, takes the
// state that the sequence starts from (its own may be written by the last segment
// while the first reads).  A thread has WIDE elements, so that many blocks have some;
// `block`: of all joining ones.
template <int D, int WIDE>
__device__ __forceinline__ void join_segments(const StateArgs &A, int block) {
  constexpr int PIECES = D * D / kThreads / WIDE, AHEAD = 32 / WIDE;
  using Wide = float __attribute__((ext_vector_type(WIDE)));
  const int h = block / PIECES % A.n_heads, lane = threadIdx.x & 63;
  int left = block / (PIECES * A.n_heads), before = 0, at_sequence = -1;  // the sequence's number among them
  for (int s0 = 0; s0 < A.n_seqs && at_sequence < 0; s0 += 64) {
    const int m = places(A, s0 + lane), took = sum_upto(m, lane);
    uint64_t some = __ballot(m > 0);
    const int count = __popcll(some);
    if (left < count) {
      for (; left; --left) some &= some - 1;
      const int at = __builtin_ctzll(some);
      at_sequence = s0 + at;
      before += __shfl(took - m, at);
    } else {
      left -= count;
      before += __shfl(took, 63);
    }
  }
  if (at_sequence < 0) return;
  const int n = places(A, at_sequence);
  if (!room_for(A, before, n)) return;
  const Sequence q = sequence(A, at_sequence);
  const int64_t D2 = (int64_t)D * D, step = A.n_heads * D2, at = (block % PIECES * kThreads + threadIdx.x) * WIDE;
  const float kept = exact_power(A, h, A.segment);
  float *const p = A.local + ((int64_t)before * A.n_heads + h) * D2 + at;
  Wide s = {};
  if (!q.fresh) s = *(const Wide *)(A.states + ((int64_t)q.state * A.n_heads + h) * D2 + at);
  *(Wide *)(p + (n - 1) * step) = s;
  for (int j = 0; j + 1 < n; j += AHEAD) {
    Wide own[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) own[i] = *(const Wide *)(p + min(j + i, n - 2) * step);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (j + i > n - 2) break;
#pragma unroll
      for (int e = 0; e < WIDE; ++e) s[e] = __builtin_fmaf(kept, s[e], own[i][e]);
      *(Wide *)(p + (j + i) * step) = s;
    }
  }
}

// ------------------------------------------------------------- token by token --
// A block has COLS columns of a head's state, a thread HELD pieces of four in rows
// ROWS apart: the state is read and written once, all of it under way at once, and
// columns need nothing of each other.  Few columns a block where heads are few, so
// that more CUs load.  64 users of 8 heads 14.9 us (4.6 TB/s; a copy 5.2), one user of
// one head 4.6, the time of a launch and of loads that wait for each other.  Blocks
// behind those of the last sequence join segments, whose own sums are there by then (of
// WIDE elements a thread; 0: none).
constexpr int kStepHeads = 8;  // query heads at a time

template <int TYPE, int D, int COLS, int WIDE>
__global__ __launch_bounds__(kThreads) void k_state_step(StateArgs A) {
  if constexpr (WIDE > 0)
    if ((int)blockIdx.y >= A.n_seqs) return join_segments<D, WIDE>(A, (blockIdx.y - A.n_seqs) * gridDim.x + blockIdx.x);
  constexpr int LANES = COLS / 4, ROWS = kThreads / LANES, HELD = D / ROWS, PARTS = D / COLS, WAVES = kThreads / 64;
  static_assert(HELD >= 1 && LANES <= 64, "a piece a thread at least, a row in a wavefront");
  __shared__ float ks[D], qs[kStepHeads][D], sums[WAVES][kStepHeads][COLS];
  const int part = blockIdx.x % PARTS, h = blockIdx.x / PARTS, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int group = A.n_q_heads / A.n_heads, row = threadIdx.x / LANES, col = threadIdx.x % LANES * 4;
  const Sequence q = sequence(A, blockIdx.y);
  if (q.count < 1 || q.count > A.step_most) return;
  float *const at = q.state < 0 ? nullptr : A.states + ((int64_t)q.state * A.n_heads + h) * D * D + part * COLS + col;
  float4v s[HELD];
#pragma unroll
  for (int i = 0; i < HELD; ++i) s[i] = q.fresh ? float4v{0, 0, 0, 0} : *(const float4v *)(at + (int64_t)(i * ROWS + row) * D);
  const float l = exact_power(A, h, 1);  // while the state is on its way
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
using float2v = float __attribute__((ext_vector_type(2)));
using half2v = _Float16 __attribute__((ext_vector_type(2)));
using half8v = _Float16 __attribute__((ext_vector_type(8)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using short4v = short __attribute__((ext_vector_type(4)));
using short8v = short __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float4v multiply(float a, float b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
template <int TYPE>
__device__ __forceinline__ float4v multiply(short8v a, short8v b, float4v c) {
  if constexpr (TYPE == kF16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Binary32 values enter a product as sums of PARTS values of its 16-bit type: what
// one alone loses (2^-9 of a value in bfloat16) an output would be off by as much
// again as by its own rounding, and a state, which is binary32, by far more.
// binary16 has no room for any binary32 value, so the values of a column of the
// operand are multiplied by a power of two that brings their largest to 2^14,
// and the result by its inverse (exactly).  Of a value far below the largest the parts
// hold fewer bits, of one below 2^-39 of it none, though it may be all that a sum has
// (where a query or a key is 0 beside the others): what they lack of it is multiplied
// by itself.  That goes by each element alone, so that no column and no token is off by
// what others hold.  (What is below 2^-140 of a column's largest has no bits behind the
// factor either and counts as 0.)
template <int TYPE, int COUNT, int PARTS>
struct Parts {
  short8v part[COUNT][PARTS];
  float factor, inverse;

  // `most`: bits of the largest magnitude of all that is multiplied by one factor.
  __device__ __forceinline__ void scale(uint32_t most) {
    const uint32_t exponent = max(most >> 23, 15u);  // at most 255
    factor = TYPE == kF16 ? __uint_as_float((268 - exponent) << 23) : 1.0f;
    inverse = TYPE == kF16 ? __uint_as_float((exponent - 14) << 23) : 1.0f;
  }
  __device__ __forceinline__ void set(const float (&x)[COUNT][8], uint32_t most) {
    scale(most);
#pragma unroll
    for (int t = 0; t < COUNT; ++t)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        float y[2] = {TYPE == kF16 ? x[t][e] * factor : x[t][e], TYPE == kF16 ? x[t][e + 1] * factor : x[t][e + 1]};
        uint32_t words[PARTS];
        split(y, words);
        put(t, e, words);
      }
  }
  // Two neighbouring values' parts; the values become what these lack of them.
  __device__ __forceinline__ static void split(float (&x)[2], uint32_t (&words)[PARTS]) {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      if constexpr (TYPE == kF16) {
        const half2v h = __builtin_convertvector((float2v{x[0], x[1]}), half2v);
        words[p] = __builtin_bit_cast(uint32_t, h);
#pragma unroll
        for (int i = 0; i < 2; ++i) x[i] = __builtin_fmaf((float)h[i], -1.0f, x[i]);  // one instruction
      } else {
        words[p] = bf16_bits(x[0]) | (uint32_t)bf16_bits(x[1]) << 16;
#pragma unroll
        for (int i = 0; i < 2; ++i) x[i] -= bf16_value((uint16_t)(words[p] >> 16 * i));
      }
    }
  }
  __device__ __forceinline__ void put(int t, int e, const uint32_t (&words)[PARTS]) {
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
      for (int i = 0; i < 2; ++i) part[t][p][e + i] = (short)(words[p] >> 16 * i);
  }
  // What the parts lack of x, of any place, behind the factor; 0 if they have all or it is
  // not small.
  __device__ __forceinline__ float rest_of_small(float x, float small) const {
    uint32_t words[PARTS];
    float rest[2] = {x * factor, 0.0f};
    const bool is_small = fabsf(rest[0]) < small;
    split(rest, words);
    return is_small ? rest[0] : 0.0f;
  }
  // x becomes what its parts lack of what is below 2^-3 behind the factor; whether that
  // is anything.
  __device__ __forceinline__ bool split_small(float (&x)[COUNT][8]) {
    bool any = false;
#pragma unroll
    for (int t = 0; t < COUNT; ++t)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        uint32_t words[PARTS];
        float y[2] = {x[t][e] * factor, x[t][e + 1] * factor};
        const bool small[2] = {fabsf(y[0]) < 0x1p-3f, fabsf(y[1]) < 0x1p-3f};
        split(y, words);
        put(t, e, words);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          x[t][e + i] = small[i] ? y[i] : 0.0f;
          any |= x[t][e + i] != 0.0f;
        }
      }
    return any;
  }
  // The least of this lane's values times the factor that is not 0.
  __device__ __forceinline__ float least(const float (&x)[COUNT][8]) const {
    uint32_t least = ~0u;  // of the bits less one: those of 0 are last
#pragma unroll
    for (int t = 0; t < COUNT; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) least = min(least, (__float_as_uint(x[t][e]) & 0x7fffffffu) - 1u);
    return least == ~0u ? __builtin_inff() : __uint_as_float(least + 1u) * factor;
  }
};

// The largest of lanes that differ in their upper two bits.
__device__ __forceinline__ uint32_t most_of_four(uint32_t x) {
  x = max(x, (uint32_t)__shfl_xor((int)x, 16));
  return max(x, (uint32_t)__shfl_xor((int)x, 32));
}
template <int TYPE, int COUNT>
__device__ __forceinline__ uint32_t largest(const float (&x)[COUNT][8]) {
  if constexpr (TYPE != kF16) return 0;
  uint32_t most = 0;
#pragma unroll
  for (int t = 0; t < COUNT; ++t)
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(x[t][e]) & 0x7fffffffu);
  return most_of_four(most);
}

// 16 bytes a lane from base + offset to LDS: the wavefront's 1024 bytes from `to`
// on, in lane order.  The compiler does not know of the load: arrive() waits.
__device__ __forceinline__ void load_to_lds(const uint8_t *base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(to) : "memory", "m0");
}
// Waits until at most LEFT of this wavefront's loads and stores are under way and
// its LDS accesses are done, then for the block's other wavefronts.
template <int LEFT>
__device__ __forceinline__ void arrive() {
  static_assert(LEFT < 16 || LEFT == 63, "a count, or all");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((LEFT & 15) | (LEFT >> 4) << 14 | 7 << 4);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// A wavefront for 16 of the values' columns.  Tiles of 64 tokens' rows lie in LDS as
// they are in memory but for the order of a row's pieces of 16 bytes: piece c of
// row r at place c ^ turn(r).
// SUMS: a segment's own sum to `local`, no outputs.  DIRECT: rows that start on
// multiples of 16 bytes go to LDS without registers, a step ahead.
template <int TYPE_, int D_, bool SUMS_, bool DIRECT_>
struct ChunkShape {
  static constexpr int TYPE = TYPE_, D = D_, WAVES = D / 16, THREADS = 64 * WAVES, PIECES = kChunk * D / 8 / THREADS;
  static constexpr bool SUMS = SUMS_, DIRECT = DIRECT_;
  static constexpr int TILE = kChunk * D;                       // 16-bit words
  // products of queries and keys, as operands in two parts: of 16 query rows with 32
  // keys, six of which are not all of later keys
  static constexpr int PART = 6 * 512, PRODUCTS = 2 * PART;
  static constexpr int KEYS = SUMS ? 4 : 2, VALUES = SUMS ? 4 : 1, QUERIES = D == 128 ? 4 : 3;  // tiles; beside them products of two heads
  static constexpr int BYTES = SUMS ? 8 * TILE * 2 : ((3 + QUERIES) * TILE + 2 * PRODUCTS) * 2;
  __device__ static __forceinline__ constexpr int product(int i, int t) { return i < 2 ? i : 2 * i - 2 + t; }

  // So that reads meet in no bank.  A transpose takes two neighbouring pieces of
  // eight rows at once: the pairs c / 2 of rows 0 to 7, and of 8 to 15, all differ.  A
  // read of 16 bytes takes 16 lanes at once, rows 0-3 and 12-15 of a piece beside
  // rows 4-11 of its neighbour (as counted of every order tried: 4 cycles a wavefront,
  // 8 with any other): rows 8-11 have the pairs of rows 4-7, the other place of each.
  // (Of 64 elements two rows lie side by side: the same of row pairs.)
  __device__ static __forceinline__ int turn(int r) {
    const int u = D == 128 ? r : r >> 1, half = D == 128 ? 8 : 4, upper = u / half & 1;
    return ((u ^ (upper * half / 2)) & (half - 1)) << 1 | upper;
  }

  // Rows [0, count) of 64 to a tile, the last one in the place of those behind it.
  __device__ static __forceinline__ void fetch(const void *from, int64_t stride, int count, short *tile) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int piece = i * THREADS + threadIdx.x, r = piece / (D / 8), c = piece % (D / 8) ^ turn(r);
      if constexpr (DIRECT) {
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        load_to_lds((const uint8_t *)from, (uint32_t)min(r, count - 1) * (uint32_t)(stride * 2) + c * 16,
                    (uint32_t)(size_t)(__attribute__((address_space(3))) short *)tile + i * THREADS * 16 + wave * 1024);
      } else {
        *(int4v *)(tile + piece * 8) = load16((const uint16_t *)from + min(r, count - 1) * stride + c * 8);
      }
    }
  }
  // An operand: a lane has row r0 + lane % 16 (r0 a multiple of 16) and columns
  // 32 t + 8 g .., g = lane / 16.  at[t]: where, in words, for r0 = 0.
  using Rows = int[D / 32];
  __device__ static __forceinline__ void places_of_rows(Rows &at) {
    const int r = threadIdx.x & 15, g = threadIdx.x >> 4 & 3;
#pragma unroll
    for (int t = 0; t < D / 32; ++t) at[t] = r * D + ((4 * t + g) ^ turn(r)) * 8;
  }
  __device__ static __forceinline__ short8v rows(const short *tile, const Rows &at, int r0, int t) {
    return *(const short8v *)(tile + at[t] + r0 * D);
  }
  // Transposes.  A lane has rows r0 + 4 g .., r0 + 16 + 4 g .. of a column: of
  // c + lane % 16 or, for the states' rows, of key_of(a, lane % 16), so that the
  // results of tiles 2 t and 2 t + 1 are in a lane what rows() gives of step t.
  __device__ static __forceinline__ constexpr int key_of(int a, int m) { return a / 2 * 32 + (m >> 2) * 8 + (a & 1) * 4 + (m & 3); }
  __device__ static __forceinline__ short8v columns_at(const short *tile, int r0, int at) {
    using Place = __attribute__((address_space(3))) short4v;
    const int r = (threadIdx.x >> 4 & 3) * 4 + (threadIdx.x >> 2 & 3);
    const short *const p = tile + r * D + ((at >> 3) ^ turn(r)) * 8 + (at & 7);
    const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Place *)(p + r0 * D));
    const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Place *)(p + (r0 + 16) * D));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  __device__ static __forceinline__ short8v columns(const short *tile, int r0, int c) { return columns_at(tile, r0, c + (threadIdx.x & 3) * 4); }
  __device__ static __forceinline__ short8v keys(const short *tile, int r0, int a) { return columns_at(tile, r0, key_of(a, (threadIdx.x & 3) * 4)); }
};
// The token of a transpose's element e in step t; results lie like that, so that they
// are operands without a move.
__device__ __forceinline__ constexpr int token(int t, int e, int g) { return t * 32 + (e >> 2) * 16 + 4 * g + (e & 3); }

// One barrier a query head: while a head's outputs are made, the next one's products
// of queries and keys are, a pair of query and key tiles a wavefront, and a later one's
// queries are loaded.  The states' columns make the wavefronts independent but for
// these products; every wavefront reads all of a head's queries from LDS, and that
// beside the products' own chain is what bounds it.  Of 4 prompts of 2048 tokens (40
// query heads over 8) 59 us, 16 of the segments' own sums, 7.7 of joining them; bytes'
// time 40.  Counted there: matrix units 34 % busy, LDS 27 %, a fifteenth of that conflicts.
// (Operands each awaited by itself 72 us, loads through registers 107, four wavefronts
// of 32 columns 107.)
template <class S>
__global__ __launch_bounds__(S::THREADS, 2) void k_state_chunk(StateArgs A) {
  constexpr int TYPE = S::TYPE, D = S::D, KT = D / 16, KS = D / 32;  // tiles and steps of a key's elements
  constexpr int TASKS = S::WAVES == 8 ? 1 : 2;                       // pairs of key tiles to a wavefront
  constexpr int PARTS = TYPE == kF16 ? 2 : 3;                        // of a decayed value: 22 or 24 bits, as the states have
  constexpr float SMALL = 0x1p-7f;  // of binary16: 2^-25 is lost of what has this or more, 2^-18 of it
  constexpr uint16_t INFINITE = TYPE == kF16 ? 0x7c00 : 0x7f80;
  extern __shared__ __attribute__((aligned(1024))) short state_lds[];
  short *const lk = state_lds, *const lv = lk + S::KEYS * S::TILE, *const lq = lv + S::VALUES * S::TILE, *const lp = lq + S::QUERIES * S::TILE;
  const Segment seg = find_segment(A, blockIdx.y);
  const int number = __builtin_amdgcn_readfirstlane(seg.number), before = __builtin_amdgcn_readfirstlane(seg.before);
  if (number < 0) return;
  Sequence q = seg.sequence;  // the block's: known to be so to the compiler as well
  q.first = __builtin_amdgcn_readfirstlane(q.first);
  q.count = __builtin_amdgcn_readfirstlane(q.count);
  q.state = __builtin_amdgcn_readfirstlane(q.state);
  q.fresh = __builtin_amdgcn_readfirstlane(q.fresh);
  if (q.count <= A.step_most) return;
  const int start = number * A.segment, tokens = min(A.segment, q.count - start), h = blockIdx.x;
  const int group = A.n_q_heads / A.n_heads, lane = threadIdx.x & 63, g = lane >> 4, own = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool last = start + tokens == q.count;
  if (S::SUMS && last) return;
  const int64_t D2 = (int64_t)D * D, row0 = q.first + start;
  float *const local = A.local + ((int64_t)(before + number) * A.n_heads + h) * D2;
  const int dv0 = wave * 16;
  // Products are made by 16 query rows and pairs of 16 keys: each SIMD (of eight
  // wavefronts w and w + 4) has two or three tiles of them.
  const int mine_i = S::WAVES == 4 ? wave : wave < 4 ? min(wave + 1, 3) : wave == 5 ? 2 : 0;
  const int mine_t = S::WAVES == 4 ? 0 : wave == 3 || wave == 5 ? 1 : wave > 5 ? 2 : 0;

  const auto fetch_k = [&](int c, int buf) {
    S::fetch((const uint16_t *)A.k + (row0 + c) * A.k_stride + h * D, A.k_stride, tokens - c, lk + buf * S::TILE);
  };
  const auto fetch_v = [&](int c, int buf) {
    S::fetch((const uint16_t *)A.v + (row0 + c) * A.v_stride + h * D, A.v_stride, tokens - c, lv + buf * S::TILE);
  };
  const auto fetch_q = [&](int c, int head, int buf) {
    S::fetch((const uint16_t *)A.q + (row0 + c) * A.q_stride + ((int64_t)h * group + head) * D, A.q_stride, tokens - c, lq + buf * S::TILE);
  };
  // The block's (chunk, head) pairs, one after another: the queries of a later one
  // are fetched while one is multiplied.
  int next_c = 0, next_head = 0, next_buf = 0;
  const auto fetch_next_q = [&] {
    if (next_c >= tokens) return false;
    fetch_q(next_c, next_head, next_buf);
    next_buf = next_buf == S::QUERIES - 1 ? 0 : next_buf + 1;
    if (++next_head == group) {
      next_head = 0;
      next_c += kChunk;
    }
    return true;
  };
  fetch_k(0, 0);
  fetch_v(0, 0);
  if constexpr (S::SUMS)  // whole chunks, as all but a sequence's last segment has
    for (int i = 1; i < 3 && i * kChunk < tokens; ++i) {
      fetch_k(i * kChunk, i);
      fetch_v(i * kChunk, i);
    }
  if constexpr (!S::SUMS) {
    for (int i = 0; i < S::QUERIES - 1; ++i) fetch_next_q();
  }

  // s[a]: rows key_of(a, 4 g) .. of column dv0 + lane % 16
  float4v s[KT] = {};
  const auto place = [&](int a, int e) { return S::key_of(a, 4 * g + e) * D + dv0 + own; };
  if constexpr (!S::SUMS) {
    const float *from = nullptr;
    // the segments' starts as join_segments leaves them
    if (number) from = local - (int64_t)A.n_heads * D2;
    else if (!q.fresh) from = last ? A.states + ((int64_t)q.state * A.n_heads + h) * D2
                                   : A.local + ((int64_t)(before + (q.count - 1) / A.segment) * A.n_heads + h) * D2;
    if (from)
#pragma unroll
      for (int a = 0; a < KT; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[a][e] = from[place(a, e)];
  }
  const Rate l2 = log2_decay(A, h);
  const float chunk_kept = exact_power(A, h, kChunk);
  // the decay between a token of this wavefront's rows and one before it
  float fade[2 * TASKS][4], row_decay = 0.0f;
  if constexpr (!S::SUMS) {
#pragma unroll
    for (int j = 0; j < 2 * TASKS; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) fade[j][e] = A.scale * power(l2, (float)max(0, (mine_i - 2 * mine_t - j) * 16 + own - 4 * g - e));
    row_decay = A.scale * power(l2, (float)(own + 1));
  }

  if constexpr (!S::SUMS) arrive<0>();
  const int out_at = own * A.n_q_heads * (D * 2) + g * 8;  // bytes; 64 rows fit 32 bits
  typename S::Rows at_rows;
  S::places_of_rows(at_rows);
  bool fetched = false, made = false;  // the last phase's queries; this chunk's first products
  int p_buf = 0;
  for (int c = 0, buf = 0, q_buf = 0; c < tokens; c += kChunk, buf = (buf + 1) & (S::KEYS - 1)) {
    const int n = S::SUMS ? kChunk : min(kChunk, tokens - c);  // a segment's own sum is of whole chunks
    const short *const k = lk + buf * S::TILE;
    const bool more = c + kChunk < tokens;
    // behind the loads of this chunk: four stores of the last one, which was whole, and later queries
    if (S::SUMS) {  // behind them the loads of up to two chunks
      if (tokens - c > 2 * kChunk) arrive<4 * S::PIECES>();
      else if (more) arrive<2 * S::PIECES>();
      else arrive<0>();
    } else if (c) {
      if (S::QUERIES > 3 && fetched) arrive<4 + S::PIECES>();
      else arrive<4>();
    }
    if (S::SUMS && c + 3 * kChunk < tokens) {
      fetch_k(c + 3 * kChunk, (buf + 3) & 3);
      fetch_v(c + 3 * kChunk, (buf + 3) & 3);
    }
    if (!S::SUMS && more) fetch_k(c + kChunk, buf ^ 1);
    short8v v[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) v[t] = S::columns(lv + (S::SUMS ? buf : 0) * S::TILE, t * 32, dv0);
    // the first token whose value in this lane's column is no number
    int none = kChunk;
    {
      using short2 = uint16_t __attribute__((ext_vector_type(2)));
      short2 most = {0, 0};
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int4v raw = __builtin_bit_cast(int4v, v[t]);
#pragma unroll
        for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(short2, raw[e] & 0x7fff7fff));
      }
      if (__any(max(most.x, most.y) >= INFINITE)) {
        // Tokens before it have a weight of 0 for it, which times it is no number: the
        // products take 0 in its place, and what sees it is made no number behind them.
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (((uint16_t)v[t][e] & INFINITE) == INFINITE) {
              none = min(none, token(t, e, g));
              v[t][e] = 0;
            }
        for (int o = 16; o < 64; o <<= 1) none = min(none, __shfl_xor(none, o));
      }
    }
    const bool numbers = !__any(none < kChunk);
    // The values' operands for the decayed products, which are bfloat16 pairs in either
    // type: a decay of a few dozen tokens leaves binary16's range.  A binary16 value
    // is the sum of two bfloat16 ones, and is not held beside them.
    constexpr bool PAIRS = TYPE == kF16 && !S::SUMS;
    short8v values[PAIRS ? 2 : 1][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      values[0][t] = v[t];
      if constexpr (PAIRS)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = value16<kF16>((uint16_t)v[t][e]);
          const uint16_t upper = bits16<kBF16>(x);
          values[0][t][e] = (short)upper;
          values[PAIRS][t][e] = (short)bits16<kBF16>(x - value16<kBF16>(upper));
        }
    }
    const auto value = [&](int t, int e) {
      if constexpr (PAIRS) return value16<kBF16>((uint16_t)values[0][t][e]) + value16<kBF16>((uint16_t)values[PAIRS][t][e]);
      else return value16<TYPE>((uint16_t)v[t][e]);
    };

    if constexpr (!S::SUMS) {
      // the state as an operand; `small`: which elements [t][e], of any lane, have less
      // than 16 bits in their parts
      Parts<TYPE, KS, 2> past;
      float past_undo[4];
      uint32_t small = 0;
      {
        float x[KS][8];
#pragma unroll
        for (int t = 0; t < KS; ++t)
#pragma unroll
          for (int e = 0; e < 8; ++e) x[t][e] = s[2 * t + (e >> 2)][e & 3];
        past.set(x, largest<TYPE, KS>(x));
#pragma unroll
        for (int e = 0; e < 4; ++e) past_undo[e] = TYPE == kF16 ? __shfl(past.inverse, 4 * g + e) : 1.0f;
        if (TYPE == kF16 && __any(past.least(x) < SMALL)) {
#pragma unroll
          for (int t = 0; t < KS; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) small |= (uint32_t)(__any(x[t][e] != 0.0f && fabsf(x[t][e] * past.factor) < SMALL) != 0) << (8 * t + e);
        }
      }
      // 16 rows of <q, k>, decayed, by pairs of 16 keys, to LDS as operands
      const auto products = [&](const short *k, const short *lq_of, int to) {
        if (2 * mine_t > mine_i) return;
        short8v mine[KS];
#pragma unroll
        for (int t = 0; t < KS; ++t) mine[t] = S::rows(lq_of + mine_i * 16 * D, at_rows, 0, t);
#pragma unroll
        for (int task = 0; task < TASKS; ++task) {
          const int t = mine_t + task;
          if (2 * t > mine_i) break;
          short8v keys[2][KS];
#pragma unroll
          for (int d = 0; d < KS; ++d)
#pragma unroll
            for (int half = 0; half < 2; ++half) keys[half][d] = S::rows(k + (2 * t + half) * 16 * D, at_rows, 0, d);
          __builtin_amdgcn_sched_barrier(0);
          float4v sum[2] = {};
#pragma unroll
          for (int d = 0; d < KS; ++d)
#pragma unroll
            for (int half = 0; half < 2; ++half) sum[half] = multiply<TYPE>(keys[half][d], mine[d], sum[half]);
          float x[1][8];
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int e = 0; e < 4; ++e)  // later tokens are left out, whatever they are
              x[0][half * 4 + e] = (2 * t + half) * 16 + 4 * g + e > mine_i * 16 + own ? 0.0f : sum[half][e] * fade[task * 2 + half][e];
          Parts<kBF16, 1, 2> p;
          p.set(x, 0);
          short *const out = lp + to * S::PRODUCTS + (S::product(mine_i, t) * 64 + lane) * 8;
          *(short8v *)out = p.part[0][0];
          *(short8v *)(out + S::PART) = p.part[0][1];
        }
      };
      // A head's outputs.  Two times two tiles of 16 rows, all of their operands on the way
      // from LDS before the first product: a wavefront that waits for each has one other to
      // wait behind.
      const auto outputs = [&](const short *lq_now, const short *lp_now, int head) {
        uint8_t *const out = (uint8_t *)A.out + (((row0 + c) * A.n_q_heads + h * group + head) * D + dv0) * 2;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (u * 32 >= n) break;
          float4v o[2] = {};
          // What the parts lack of small elements, four rows of the state at a time; other
          // elements add 0.  (Random states have one in a chunk of a hundred: with all of
          // its column in binary32 instead four prompts of 2048 tokens took 14 us longer.)
          if (PAIRS && __builtin_expect(small != 0, 0)) {
#pragma unroll
            for (int t = 0; t < KS; ++t) {
              if (!(small >> 8 * t & 0xff)) continue;
              short8v y[2];
#pragma unroll
              for (int i = 0; i < 2; ++i) y[i] = S::rows(lq_now, at_rows, u * 32 + i * 16, t);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                if (!(small >> (8 * t + e) & 1)) continue;
                float element = s[2 * t + (e >> 2)][e & 3];
                asm volatile("" : "+v"(element));  // else the rests are made before the heads, and held
                const float rest = past.rest_of_small(element, SMALL);
#pragma unroll
                for (int i = 0; i < 2; ++i) o[i] = multiply(rest, value16<TYPE>((uint16_t)y[i][e]), o[i]);
              }
            }
          }
          short8v x[2][KS], w[2][2][2];
#pragma unroll
          for (int t = 0; t < KS; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) x[i][t] = S::rows(lq_now, at_rows, u * 32 + i * 16, t);
#pragma unroll
          for (int t = 0; t <= u; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int p = 0; p < 2; ++p) w[i][t][p] = *(const short8v *)(lp_now + p * S::PART + (S::product(u * 2 + i, t) * 64 + lane) * 8);
          __builtin_amdgcn_sched_barrier(0);
          float4v near[2] = {};
          // of this chunk's tokens, without the lower parts of both (2^-18 of a product)
          const auto products_of_values = [&](float4v (&sum)[2]) {
#pragma unroll
            for (int t = 0; t <= u; ++t)
#pragma unroll
              for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int d = 0; d < (PAIRS ? 2 - p : 1); ++d)
#pragma unroll
                  for (int i = 0; i < 2; ++i) sum[i] = multiply<kBF16>(values[d][t], w[i][t][p], sum[i]);
          };
          if constexpr (PAIRS) products_of_values(near);  // beside the state's
#pragma unroll
          for (int t = 0; t < KS; ++t)
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
              for (int i = 0; i < 2; ++i) o[i] = multiply<TYPE>(past.part[t][p], x[i][t], o[i]);
          if constexpr (PAIRS) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[i][e] *= past_undo[e];
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float seen = row_decay * power(l2, (float)(u * 32 + i * 16));
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] = PAIRS ? __builtin_fmaf(o[i][e], seen, near[i][e]) : o[i][e] * seen;
          }
          if constexpr (!PAIRS) products_of_values(o);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = u * 32 + i * 16 + own;
            if (!numbers) {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (row >= __shfl(none, 4 * g + e)) o[i][e] = __builtin_nanf("");
            }
            if (row < n) {
              uint16_t bits[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) bits[e] = bits16<TYPE>(o[i][e]);
              __builtin_memcpy(out + (uint32_t)(out_at + (u * 32 + i * 16) * A.n_q_heads * (D * 2)), bits, 8);
            }
          }
        }
      };
      // The first head's products, then each head's outputs beside the next one's
      // products; beside the last one's the next chunk's first, whose keys are there two
      // phases after they were asked for.  The next chunk's values are asked for behind
      // a barrier, when all have this one's.
      const bool early = more && group >= 3;
      if (!made) {
        products(k, lq + q_buf * S::TILE, p_buf);
        arrive<63>();
        if (more) fetch_v(c + kChunk, 0);
      }
      for (int head = 0; head < group; ++head) {
        const short *const lq_now = lq + q_buf * S::TILE, *const lp_now = lp + p_buf * S::PRODUCTS;
        q_buf = q_buf == S::QUERIES - 1 ? 0 : q_buf + 1;
        const bool next_values = made && head == 1 && more;
        if (next_values) fetch_v(c + kChunk, 0);
        fetched = fetch_next_q();
        // (One wavefront of a SIMD before its outputs, the other behind them.)
        const bool ahead = head + 1 < group || early;
        const short *const k_next = head + 1 < group ? k : lk + (buf ^ 1) * S::TILE;
        if (ahead && wave < 4) products(k_next, lq + q_buf * S::TILE, p_buf ^ 1);
        outputs(lq_now, lp_now, head);
        if (ahead && wave >= 4) products(k_next, lq + q_buf * S::TILE, p_buf ^ 1);
        // The next one's products need the queries after it: behind them what this
        // one has asked for, and its stores.
        if (head + 1 < group) {
          if (n < kChunk) arrive<0>();
          else if (S::QUERIES == 3) arrive<4>();
          else if (head == 0 && more && !made) fetched ? arrive<4 + 3 * S::PIECES>() : arrive<4 + 2 * S::PIECES>();
          else if ((head == 0 && more) || next_values) fetched ? arrive<4 + 2 * S::PIECES>() : arrive<4 + S::PIECES>();
          else fetched ? arrive<4 + S::PIECES>() : arrive<4>();
        }
        p_buf ^= 1;
      }
      made = early;
      if (last && q.state < 0 && !more) return;
    }
    // the state after the chunk
    const float kept = n == kChunk ? chunk_kept : exact_power(A, h, n);
    Parts<TYPE, 1, PARTS> fading[2];  // 32 tokens each: a factor for both would be the last ones'
    float x[2][1][8];
    {
      const float behind = (float)(n - 1 - 4 * g);  // tokens, of the chunk's behind this lane's first
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          x[t][0][e] = value(t, e) * power(l2, behind - (float)token(t, e, 0));
      if (n < kChunk) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (token(t, e, g) >= n) x[t][0][e] = 0.0f;
      }
      if (!numbers) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (token(t, e, g) == none) x[t][0][e] = __builtin_nanf("");
      }
    }
    bool some = false;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      fading[t].scale(largest<TYPE, 1>(x[t]));
      some |= fading[t].split_small(x[t]);
    }
    short8v keys[KT][2];
#pragma unroll
    for (int a = 0; a < KT; ++a)
#pragma unroll
      for (int t = 0; t < 2; ++t) keys[a][t] = S::keys(k, t * 32, a);
    __builtin_amdgcn_sched_barrier(0);
    for (float held = kept;; held = 1.0f) {
#pragma unroll
      for (int a = 0; a < KT; a += 4) {  // four sums side by side, none waits for itself
        if constexpr (TYPE == kF16) {
          float4v sum[2][4] = {};
#pragma unroll
          for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int i = 0; i < 4; ++i) sum[t][i] = multiply<TYPE>(keys[a + i][t], fading[t].part[0][p], sum[t][i]);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s[a + i][e] = __builtin_fmaf(sum[1][i][e], fading[1].inverse, __builtin_fmaf(sum[0][i][e], fading[0].inverse, s[a + i][e] * held));
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) s[a + i] *= held;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
              for (int i = 0; i < 4; ++i) s[a + i] = multiply<TYPE>(keys[a + i][t], fading[t].part[0][p], s[a + i]);
        }
      }
      // What two binary16 parts lack of values of which they hold less than 22 bits, 2^-25
      // at most, goes in behind a factor of its own as often as there is any: four times at
      // most, then no bit of binary32 is left.  (Decays that leave 2^-14 of a value in 32
      // tokens need none but for a few values, faster ones one or two: 4 prompts of 4096
      // tokens, 16 heads of 128 from exp(-0.7) to exp(-0.004) a token, 179 us, all at
      // exp(-0.004) 155, 136 where small values are lost.  With all of the column in binary32
      // instead the first took 321.)
      if (TYPE != kF16 || !__any(some)) break;
      some = false;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        fading[t].factor = 0x1p39f;
        fading[t].inverse *= 0x1p-39f;
        some |= fading[t].split_small(x[t]);
      }
    }
  }
  float *to = nullptr;
  if constexpr (S::SUMS) to = local;
  else if (last && q.state >= 0) to = A.states + ((int64_t)q.state * A.n_heads + h) * D2;
  if (to)
#pragma unroll
    for (int a = 0; a < KT; ++a)
#pragma unroll
      for (int e = 0; e < 4; ++e) to[place(a, e)] = s[a][e];
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

// Blocks of outputs at once: a CU has one at head_dim 128, two at 64.
int64_t blocks_at_once(int32_t head_dim) { return head_dim == 128 ? 256 : 512; }

// The least tokens of a segment: so many that all tokens make about a segment of a
// head for each of those.
int segment_least(int64_t n_tokens, int64_t n_heads, int32_t head_dim) {
  const int64_t blocks = blocks_at_once(head_dim), L = ((n_tokens * n_heads + blocks - 1) / blocks + kChunk - 1) / kChunk * kChunk;
  return (int)std::max<int64_t>(kChunk, std::min<int64_t>(L, 1 << 30));
}

// Tokens of a segment, that many or more: those that take least if one sequence has
// max_q new tokens and the others share what is left (where that is no more than
// kStepMost each, the long one is alone).  Times in us of what is measured at head_dim
// 128: 2.2 for a chunk and query head, 1.5 for a chunk beside, 2 for a chunk of a
// segment's sum, what launches and starts take; a segment a sequence needs no sums.
// Sequences of one length are whole rounds of blocks; of others half a segment each is
// left over, and blocks behind the first round fill up what is free.  (Lengths in
// eighths of the least: 6 prompts of 17211 tokens, 8 heads of 128, 422 us, 553 where
// only its halves are tried; 27 of up to 15696 tokens, 6 heads of 64 over 3, 169, and
// 235 as equal ones.)
int segment_tokens(const StateArgs &A) {
  const int64_t least = segment_least(A.n_tokens, A.n_heads, A.head_dim), longest = (A.max_q + kChunk - 1) / kChunk * kChunk;
  const double slots = (double)blocks_at_once(A.head_dim), chunk = 1.5 + 2.2 * (A.n_q_heads / A.n_heads);
  const double other = A.n_seqs > 1 ? std::min<double>(A.max_q, (double)(A.n_tokens - A.max_q) / (A.n_seqs - 1)) : 0.0;
  const double others = other > kStepMost ? A.n_seqs - 1 : 0;
  const bool equal = others == 0 || other == A.max_q;
  const auto time = [&](int64_t L) {
    const double parts = (double)((A.max_q + L - 1) / L), chunks = (double)(std::min(L, longest) / kChunk);
    const double blocks = A.n_heads * (parts + others * (equal ? parts : std::max(1.0, other / (double)L + 0.5)));
    const double whole = A.n_heads * ((double)A.max_q + others * other) / (double)(chunks * kChunk);
    const double rounds = blocks <= slots ? 1.0 : equal ? std::ceil(blocks / slots) : whole / slots + 0.8;
    return rounds * (chunks * chunk + 6.0) + (parts > 1 ? rounds * (chunks * 2.0 + 5.0) + 6.0 : 0.0);
  };
  int64_t best = least;
  const int64_t step = std::max<int64_t>(1, least / 8 / kChunk) * kChunk;
  for (int i = 1; i <= 28; ++i) {
    const int64_t L = i < 28 ? least + i * step : longest;
    if (L >= least && time(L) < time(best)) best = L;
  }
  return (int)std::min<int64_t>(best, 1 << 30);
}
// Places of sequences of more than a segment's L tokens: n of them have less than
// n / L + 1 segments, and so many sequences n / L at most.  L is the least length's
// multiple of kChunk, so n / L goes down where that goes up; it is no more than that of
// the least length itself and of kChunk, which grow with n.
int64_t places_at_most(int64_t n_tokens, int64_t n_heads, int32_t head_dim, int64_t n_seqs) {
  const int64_t most = std::min<int64_t>(n_tokens / kChunk, blocks_at_once(head_dim) / n_heads);
  return n_tokens > kChunk ? most + std::min(n_seqs, most) : 0;
}

template <class S>
hipError_t chunks_as(dim3 grid, const StateArgs &A, hipStream_t s) {
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_state_chunk<S>), hipFuncAttributeMaxDynamicSharedMemorySize, S::BYTES);
  if (e != hipSuccess) return e;
  k_state_chunk<S><<<grid, S::THREADS, S::BYTES, s>>>(A);
  return hipGetLastError();
}

template <int TYPE, int D, bool SUMS>
hipError_t chunks_of(dim3 grid, const StateArgs &A, hipStream_t s) {
  // rows that start on multiples of 16 bytes, 64 of them within 32 bits
  const auto whole = [](const void *p, int64_t stride) { return (((uintptr_t)p | (uintptr_t)(stride * 2)) & 15) == 0 && stride <= 1 << 24; };
  if (whole(A.k, A.k_stride) && whole(A.v, A.v_stride) && (SUMS || whole(A.q, A.q_stride)))
    return chunks_as<ChunkShape<TYPE, D, SUMS, true>>(grid, A, s);
  return chunks_as<ChunkShape<TYPE, D, SUMS, false>>(grid, A, s);
}

template <int TYPE, int D, int COLS, int WIDE>
hipError_t steps_as(const StateArgs &A, int64_t joined, hipStream_t s) {
  const int64_t width = (int64_t)A.n_heads * (D / COLS);
  const int64_t joins = WIDE ? joined * A.n_heads * (D * D / kThreads / std::max(WIDE, 1)) : 0;
  k_state_step<TYPE, D, COLS, WIDE><<<dim3((unsigned)width, (unsigned)(A.n_seqs + (joins + width - 1) / width)), kThreads, 0, s>>>(A);
  return hipGetLastError();
}
// Single tokens, and behind them `joined` sequences' segments to be joined.
// (Joining 128 segments of 2 heads takes 24 us with four elements a thread, 11 with
// one; 8 of 32 heads 7.5 and 12, where blocks are many.)
template <int TYPE, int D>
hipError_t steps_of(const StateArgs &A, int64_t joined, hipStream_t s) {
  const int64_t heads = (int64_t)A.n_seqs * A.n_heads;
  if (joined) return joined * A.n_heads >= 16 ? steps_as<TYPE, D, 32, 4>(A, joined, s) : steps_as<TYPE, D, 16, 1>(A, joined, s);
  if (heads >= 512) return steps_as<TYPE, D, D, 0>(A, 0, s);
  if (heads >= 128) return steps_as<TYPE, D, 32, 0>(A, 0, s);
  return steps_as<TYPE, D, 16, 0>(A, 0, s);
}

template <int TYPE, int D>
hipError_t state_of(StateArgs A, hipStream_t s) {
  A.max_q = std::min(A.max_q, A.n_tokens);
  A.segment = segment_tokens(A);
  A.n_places = (int32_t)places_at_most(A.n_tokens, A.n_heads, A.head_dim, A.n_seqs);
  A.step_most = kStepMost;
  if (A.max_q <= kStepMost) return steps_of<TYPE, D>(A, 0, s);
  if (A.n_seqs == 1) A.step_most = 0;  // no launch for what may be a single token
  const bool one = A.segment >= A.max_q;  // a segment a sequence
  // Heads first: blocks that find no segment come last.  (Between the others they left
  // them to half of the CUs: one prompt of 12260 tokens beside 15 single ones, 12 heads,
  // 148 us of the outputs instead of 92.)  No more than blocks_at_once segments and a sequence's
  // last, see segment_least.
  const dim3 grid(A.n_heads, one ? (unsigned)A.n_seqs : (unsigned)(A.n_tokens / A.segment + A.n_seqs));
  hipError_t e = one ? hipSuccess : chunks_of<TYPE, D, true>(grid, A, s);
  // at most so many sequences have more tokens than a segment
  const int64_t joined = one ? 0 : std::min<int64_t>(A.n_seqs, A.n_tokens / A.segment);
  if (e == hipSuccess && (joined || A.step_most)) e = steps_of<TYPE, D>(A, joined, s);
  return e == hipSuccess ? chunks_of<TYPE, D, false>(grid, A, s) : e;
}

}  // namespace

size_t state_workspace(int32_t n_heads, int32_t head_dim, int64_t n_tokens, int32_t n_seqs) {
  return (size_t)(places_at_most(n_tokens, n_heads, head_dim, n_seqs) * n_heads * head_dim * head_dim) * 4;
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
