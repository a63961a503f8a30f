// fs_product.h -- the kernels of projections in 8-bit integers and what chooses
// among them: rows of activations to codes with a scale a row, behind an RMS norm
// or not, and the product of codes with weights that have a scale an output
// channel.  A file that includes it makes the kernels that it launches.
//
// y[m][n] = (sum_k a[m][k] w[n][k]) * a_scale[m] * w_scale[n] + bias[n].
// The sum is exact in 32-bit integers whatever the order, so tiles, splits
// and instructions are free to choose and every variant gives the same bits.
//
// In all variants the weights are the instruction's first operand, so a
// lane's four results are neighbouring channels of one token.
#pragma once

#include <algorithm>

#include "fs_serving.h"

namespace fs {
namespace {

// The largest |x| of a block's values by their bit patterns: a NaN is larger
// than an infinity, so neither is lost in the maximum.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// A wavefront's sum or largest, in every lane: rows of 16 by shifts within them, the
// rows by two broadcasts (lanes that get nothing take 0), the last lane's to all.
template <int CONTROL, int ROWS>
__device__ __forceinline__ uint32_t from_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, ROWS, 0xf, true);
}
template <class Join>
__device__ __forceinline__ uint32_t join_wave(uint32_t v, Join join) {
  v = join(v, from_lane<0x111, 0xf>(v));  // by 1, 2, 4, 8
  v = join(v, from_lane<0x112, 0xf>(v));
  v = join(v, from_lane<0x114, 0xf>(v));
  v = join(v, from_lane<0x118, 0xf>(v));
  v = join(v, from_lane<0x142, 0xa>(v));  // the last of rows 0 and 2 to rows 1 and 3
  v = join(v, from_lane<0x143, 0xc>(v));  // of row 1 to rows 2 and 3
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  return join_wave(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
  return __uint_as_float(join_wave(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

template <int THREADS>
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t *lds) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
  for (int i = 1; i < THREADS / 64; ++i) v = max(v, lds[i]);
  return v;
}

// Eight neighbouring elements of a row from c <= cols on, zeros from `cols` on;
// `whole`: rows start on multiples of 16 bytes.  (c + 8 may have no 32 bits.)
template <int TYPE>
__device__ __forceinline__ void load8_of(const void *x, int64_t row, int c, int cols, bool whole, float (&v)[8]) {
  if (cols - c >= 8) {
    load8<TYPE>(x, row + c, whole, v);
  } else if (c < cols) {  // all loads under way together, the last element's in the place of those behind it
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = load_value<TYPE>(x, row + c + min(i, cols - c - 1));
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= cols - c) v[i] = 0.0f;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
  }
}

// Eight codes: x * inverse (of at most 127) to the nearest whole number, ties to
// even, by the addition of 1.5 * 2^23, whose result holds it in its low byte.
__device__ __forceinline__ int2 codes8(const float (&v)[8], float inverse) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i] * inverse + 12582912.0f);
  int word[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    word[i] = (int)__builtin_amdgcn_perm(__builtin_amdgcn_perm(w[4 * i + 3], w[4 * i + 2], 0x0c0c0400),
                                         __builtin_amdgcn_perm(w[4 * i + 1], w[4 * i], 0x0c0c0400), 0x05040100);
  return {word[0], word[1]};
}

__device__ __forceinline__ void store_codes8(int8_t *out, int c, int cols, const float (&v)[8], float inverse) {
  const int2 word = codes8(v, inverse);
  if (cols - c >= 8) {
    __builtin_memcpy(out + c, &word, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < cols - c) out[c + i] = (int8_t)((i < 4 ? word.x : word.y) >> (8 * (i & 3)));
  }
}

// The mean of squares that an RMS norm divides by, of any finite values: two
// sums, of x^2 and of (2^-80 x)^2, the second where the first may pass what
// binary32 holds (131071 of the largest values make 2^113 of it).  (What the first loses below 2^-126 is of no account beside an
// eps of 2^-80 at least.)
struct Squares {
  float sum, low;

  __device__ __forceinline__ void add(float x) {
    const float y = x * 0x1p-80f;
    sum = __builtin_fmaf(x, x, sum);
    low = __builtin_fmaf(y, y, low);
  }
  __device__ __forceinline__ void add(const Squares &o) {
    sum += o.sum;
    low += o.low;
  }
  __device__ __forceinline__ void join_lanes() {
    sum = wave_sum(sum);
    low = wave_sum(low);
  }
  // 1 / sqrt(mean + eps), by v_rsq_f32: within a step
  __device__ __forceinline__ float factor(int count, float eps) const {
    if (sum < 0x1p100f) return __builtin_amdgcn_rsqf(sum / (float)max(count, 1) + eps);
    return 0x1p-80f * __builtin_amdgcn_rsqf(low / (float)count + eps * 0x1p-160f);
  }
};

// Eight neighbouring gains from c on (`cols` of them, ones if there are none).
__device__ __forceinline__ void gain8(const float *gain, int c, int cols, float (&g)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] = 1.0f;
  if (gain) load8_of<kF32>(gain, 0, c, cols, true, g);
}

// One block a row, the row in registers: HELD groups of 8 elements a thread.
// HELD = 0: a row too long for that is read twice (the second time from L2).
// NORMED: the row's RMS norm first.  Its factor 1 / sqrt(mean x^2 + eps) is the
// row's and cancels in the codes, which are those of x * gain: it goes into the
// scale alone, and the row is read once.
template <int TYPE, int THREADS, int HELD, bool NORMED>
__global__ __launch_bounds__(THREADS) void k_quantize_rows(QuantizeArgs A) {
  __shared__ uint32_t lds[THREADS / 64];
  __shared__ Squares squares[NORMED ? THREADS / 64 : 1];
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < A.n_zero; i += THREADS) A.zero[i] = 0;
  Squares mine = {0.0f, 0.0f};
  const auto norm = [&](const float(&g)[8], float(&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      mine.add(x[i]);
      x[i] *= g[i];
    }
  };
  const int64_t row = blockIdx.x, at = row * A.x_stride;
  const int own = threadIdx.x * 8, step = THREADS * 8;
  const bool whole = (((uintptr_t)A.x | (uintptr_t)(A.x_stride * 2)) & 15) == 0;
  float v[HELD ? HELD : 1][8];
  uint32_t most = 0;
  if constexpr (HELD > 0) {
    float gains[NORMED ? HELD : 1][8];  // on the way with the row
    if constexpr (NORMED) {
#pragma unroll
      for (int j = 0; j < HELD; ++j) gain8(A.gain, min(own + j * step, A.cols), A.cols, gains[j]);
    }
#pragma unroll
    for (int j = 0; j < HELD; ++j) load8_of<TYPE>(A.x, at, min(own + j * step, A.cols), A.cols, whole, v[j]);
    if constexpr (NORMED) {
#pragma unroll
      for (int j = 0; j < HELD; ++j) norm(gains[j], v[j]);
    }
#pragma unroll
    for (int j = 0; j < HELD; ++j)
      for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[j][i]));
  } else {
    for (int64_t c = own; c < A.cols; c += step) {
      load8_of<TYPE>(A.x, at, (int)c, A.cols, whole, v[0]);
      if constexpr (NORMED) {
        float g[8];
        gain8(A.gain, (int)c, A.cols, g);
        norm(g, v[0]);
      }
      for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[0][i]));
    }
  }
  if constexpr (NORMED) {
    mine.join_lanes();
    if ((threadIdx.x & 63) == 0) squares[threadIdx.x >> 6] = mine;
  }
  const float a = __uint_as_float(block_max<THREADS>(most, lds));
  float factor = 1.0f;
  if constexpr (NORMED) {  // all wavefronts' squares are there
    mine = squares[min((int)threadIdx.x & 63, THREADS / 64 - 1)];
    if ((threadIdx.x & 63) >= THREADS / 64) mine = {0.0f, 0.0f};
    mine.join_lanes();
    factor = mine.factor(A.cols, A.eps);
  }
  const bool zero = a < kTiny;
  const float inverse = zero ? 0.0f : 127.0f / a;
  int8_t *const out = A.codes + row * A.code_stride;
  if constexpr (HELD > 0) {
#pragma unroll
    for (int j = 0; j < HELD; ++j)
      if (own + j * step < A.cols) store_codes8(out, own + j * step, A.cols, v[j], inverse);
  } else {
    for (int64_t c = own; c < A.cols; c += step) {
      load8_of<TYPE>(A.x, at, (int)c, A.cols, whole, v[0]);
      if constexpr (NORMED) {
        float g[8];
        gain8(A.gain, (int)c, A.cols, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[0][i] *= g[i];
      }
      store_codes8(out, (int)c, A.cols, v[0], inverse);
    }
  }
  if (threadIdx.x == 0) A.scale[row] = zero ? 0.0f : (NORMED ? a * factor : a) / 127.0f;
}

// 16 codes of a row (of K > 0) from column k on.  load() only asks for the
// words, so that loads follow one another; codes() waits and shifts.  A stage
// that passes the row's end (`over`) takes the row's last 16, and shifts zeros
// in.
struct Piece {
  Words words;

  __device__ __forceinline__ void load(const int8_t *row, int k, int K, bool over) {
    if (!over) {
      words.load(row + k);
    } else if (K >= 16) {
      words.load(row + min(k, K - 16));
    } else {  // a short row: byte by byte
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 15; ++i)
        if (i < K) w[i >> 2] |= (uint32_t)(uint8_t)row[i] << 8 * (i & 3);
      words.set(int4v{(int)w[0], (int)w[1], (int)w[2], (int)w[3]});
    }
  }
  __device__ __forceinline__ int4v codes(int k, int K, bool over) const {
    const int4v v = words.value();
    if (!over) return v;
    const int beyond = k - max(0, min(k, K - 16));
    const unsigned __int128 w = __builtin_bit_cast(unsigned __int128, v);
    return __builtin_bit_cast(int4v, beyond < 16 ? w >> beyond * 8 : (unsigned __int128)0);
  }
};

// Four neighbouring channels from n (a multiple of 4) on of token m.
template <int TYPE>
__device__ __forceinline__ void store_products(const MatmulArgs &A, int m, int n, int4v acc, float sa, float4v sw,
                                               float4v bias) {
  const int64_t at = (int64_t)m * A.out_stride + n;
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = (float)acc[i] * sa * sw[i];
    if (A.bias) y[i] += bias[i];
  }
  if (A.N - n >= 4) {  // one store at any alignment
    if constexpr (TYPE == kF32) {
      __builtin_memcpy((float *)A.out + at, y, 16);
    } else {
      uint16_t h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = bits16<TYPE>(y[i]);
      __builtin_memcpy((uint16_t *)A.out + at, h, 8);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < A.N - n) store_value<TYPE>(A.out, at + i, y[i]);
  }
}

// -------------------------------------------------------- tiles through LDS --
// Tiles of BM tokens x BN channels, BK inner elements a stage, a ring of NS
// stages in LDS, all but one of them in flight while one is multiplied.  Loads
// go straight to LDS, where a lane's place is fixed, so the lanes' addresses
// carry the order: a row of BK bytes is BK / 16 chunks, chunk c of row r at
// place c ^ turn(r), so that the 16 rows that a quarter of a wavefront reads
// fall on all 64 banks.
template <int BK>
__device__ __forceinline__ int turn(int r) {
  if constexpr (BK >= 256) return r & 15;
  else if constexpr (BK == 128) return (r >> 1) & 7;
  else return (r >> 2) & 3;
}

// 16 bytes a lane from base + offset to LDS: the wavefront's 1024 bytes from
// `to` on, in lane order.  Counted like any load; the compiler does not know
// of it, so arrive() waits.
__device__ __forceinline__ void load_to_lds(const int8_t *base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(to) : "memory", "m0");
}

// Waits until at most LOADS of this wavefront's loads are under way and its
// LDS reads are done.
template <int LOADS>
__device__ __forceinline__ void wait_loads() {
  static_assert(LOADS < 64, "the counter has 6 bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((LOADS & 15) | (LOADS >> 4) << 14 | 7 << 4);
}

// The same for a ring of NS stages of L loads each when `after` stages beyond
// the wanted one are under way: the largest of a few counts that is enough.
template <int NS, int L>
__device__ __forceinline__ void wait_stage(int after) {
  if (after >= NS - 2) wait_loads<(NS - 2) * L>();
  else if (NS > 4 && after >= NS / 2) wait_loads<NS / 2 * L>();
  else if (NS > 6 && after >= NS / 4) wait_loads<NS / 4 * L>();
  else wait_loads<0>();
}

template <int TYPE_, int BM_, int BN_, int WM_, int WN_, int BK_, int WK_, int NS_>
struct Shape {
  static constexpr int TYPE = TYPE_, BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = BK_, NS = NS_;
  // WK wavefronts share a part of the tile, each with its part of a stage:
  // fewer, longer stages, where waiting for each is what costs
  static constexpr int WK = WK_, TILES = (BM / WM) * (BN / WN);
  static constexpr int WAVES = TILES * WK, THREADS = 64 * WAVES, MT = WM / 16, NT = WN / 16, CH = BK / 16;
  static constexpr int LA = BM * CH / THREADS, LW = BN * CH / THREADS;  // loads of a thread a stage
  static constexpr int PART_A = BM * BK, STAGE = (BM + BN) * BK, BYTES = NS * STAGE;
  static_assert(BK % (64 * WK) == 0, "a part of a stage is whole steps");
  static_assert(WK == 1 || WAVES * MT * NT * 1024 <= BYTES, "the parts' sums fit the ring");
  static_assert(LA * THREADS == BM * CH && LW * THREADS == BN * CH && LA > 0 && LW > 0, "whole loads");
};

// What a product ends in: scales and a bias; beside these an activation and the
// residual stream; or, of gate and value channels, the product of the activated
// gate and the value.
enum Finish { kScaled, kFinished, kGated };

// A gated tile of BN / 2 channels has both weight rows of each, so placed that
// one lane gets both sums: a wavefront's rows are its channels' gates, then their
// values; of 16 rows every two gates are followed by their two values.
struct WeightRow {
  int channel;
  bool value;
};
template <class S, Finish FINISH>
__device__ __forceinline__ WeightRow weight_row(int r) {
  if constexpr (FINISH != kGated) return {r, false};
  const int in = r % S::WN, from = r / S::WN * (S::WN / 2);
  if constexpr (S::NT == 1) return {from + (in >> 2) * 2 + (in & 1), (in & 2) != 0};
  else return {from + in % (S::WN / 2), in >= S::WN / 2};
}
template <class S, Finish FINISH>
constexpr int kChannels = FINISH == kGated ? S::BN / 2 : S::BN;

template <class S>
__device__ __forceinline__ void multiply_stage(const int8_t *la, const int8_t *lw, int wm, int wn, int wk, int lane,
                                               int4v (&acc)[S::MT][S::NT]) {
  constexpr int STEPS = S::BK / 64 / S::WK;
#pragma unroll
  for (int kk = 0; kk < STEPS; ++kk) {
    int4v fa[S::MT], fw[S::NT];
    const int r = lane & 15, at = (((wk * STEPS + kk) * 4 + (lane >> 4)) ^ turn<S::BK>(r)) * 16;  // rows differ by multiples of 16
#pragma unroll
    for (int i = 0; i < S::MT; ++i) fa[i] = *(const int4v *)(la + (wm + i * 16 + r) * S::BK + at);
#pragma unroll
    for (int j = 0; j < S::NT; ++j) fw[j] = *(const int4v *)(lw + (wn + j * 16 + r) * S::BK + at);
#pragma unroll
    for (int i = 0; i < S::MT; ++i)
#pragma unroll
      for (int j = 0; j < S::NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[j], fa[i], acc[i][j], 0, 0, 0);
  }
}

// Row and first inner element of a thread's i-th place in a part of a stage.
template <class S>
__device__ __forceinline__ int2 place(int i) {
  const int slot = i * S::THREADS + threadIdx.x, r = slot / S::CH;
  return {r, (slot % S::CH ^ turn<S::BK>(r)) * 16};
}

// The sums of the wavefronts that share a tile meet in LDS, each tile at its
// first one; the others are done.
template <class S>
__device__ __forceinline__ bool join_parts(int8_t *lds, int wk, int wave, int lane, int4v (&acc)[S::MT][S::NT]) {
  if constexpr (S::WK > 1) {
    __syncthreads();
    int4v *const sums = (int4v *)lds;
#pragma unroll
    for (int i = 0; i < S::MT; ++i)
#pragma unroll
      for (int j = 0; j < S::NT; ++j) sums[(wave * S::MT * S::NT + i * S::NT + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    if (wk > 0) return false;
#pragma unroll
    for (int i = 0; i < S::MT; ++i)
#pragma unroll
      for (int j = 0; j < S::NT; ++j)
        for (int p = 1; p < S::WK; ++p)
          acc[i][j] += sums[((p * S::TILES + wave) * S::MT * S::NT + i * S::NT + j) * 64 + lane];
  }
  return true;
}

// The sums of the blocks that share a tile meet in memory: each writes its own, and
// the last to arrive adds the others' (whole numbers: the order is of no account).
// They go from block to block, whose L2 may be another XCD's, at the device's scope,
// past the L2.  True: of the last one.
template <class S>
__device__ __forceinline__ bool join_blocks(const MatmulArgs &A, int slot, int part, int parts, bool mine, int wt, int lane,
                                            int4v (&acc)[S::MT][S::NT]) {
  __shared__ int last;
  constexpr int COUNT = S::MT * S::NT, LANES = S::TILES * 64;
  using Two = unsigned long long;
  Two *const sums = (Two *)A.partials + ((int64_t)slot * parts * COUNT * LANES + wt * 64 + lane) * 2;
  const auto at = [&](int p, int c) { return sums + ((int64_t)p * COUNT + c) * LANES * 2; };
  if (mine) {
#pragma unroll
    for (int c = 0; c < COUNT; ++c) {
      const int4v v = acc[c / S::NT][c % S::NT];
      __hip_atomic_store(at(part, c), (Two)(uint32_t)v[0] | (Two)(uint32_t)v[1] << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(at(part, c) + 1, (Two)(uint32_t)v[2] | (Two)(uint32_t)v[3] << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // each wavefront's stores are done before the block counts as there
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(A.arrived + slot, 1) == parts - 1;
  __syncthreads();
  if (!last) return false;
  if (mine)
    for (int p = 0; p < parts; ++p) {
      if (p == part) continue;
#pragma unroll
      for (int c = 0; c < COUNT; ++c) {
        const Two a = __hip_atomic_load(at(p, c), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const Two b = __hip_atomic_load(at(p, c) + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        acc[c / S::NT][c % S::NT] += int4v{(int)(uint32_t)a, (int)(a >> 32), (int)(uint32_t)b, (int)(b >> 32)};
      }
    }
  return true;
}

// A wavefront's part of a tile, from token m and channel n on.
template <class S>
__device__ __forceinline__ void store_tile(const MatmulArgs &A, int m, int n, int lane, int4v (&acc)[S::MT][S::NT],
                                           const float (&sa)[S::MT]) {
  // the scales first, all loads under way together
  float4v sw[S::NT], bias[S::NT];
  const auto channels = [&](const float *from, float4v (&to)[S::NT]) {
#pragma unroll
    for (int j = 0; j < S::NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) to[j][i] = from[min(n + j * 16 + (lane >> 4) * 4 + i, A.N - 1)];
  };
  channels(A.w_scale, sw);
  if (A.bias) channels(A.bias, bias);
#pragma unroll
  for (int i = 0; i < S::MT; ++i) {
    const int row = m + i * 16 + (lane & 15);
#pragma unroll
    for (int j = 0; j < S::NT; ++j) {
      const int channel = n + j * 16 + (lane >> 4) * 4;
      if (row < A.M && channel < A.N) store_products<S::TYPE>(A, row, channel, acc[i][j], sa[i], sw[j], bias[j]);
    }
  }
}

// An activation of four values.  Exponentials by v_exp_f32 and reciprocals by
// v_rcp_f32, each within a step of binary32; the exponent's rounding moves a
// sigmoid at t by up to 2^-24 |t| of itself.  gelu: (1 - erf z) / 2 at z = |x| / sqrt 2
// is exp(-z^2) and what falls as 1 / z, a polynomial in t = 1 / (1 + 0.44 z) without
// a constant, fitted to it over z <= 10 within 2e-7 of itself: the value of a negative x
// is as good as that of a positive one.
__device__ __forceinline__ float exp_of(float t) { return __builtin_amdgcn_exp2f(t * 1.44269504f); }

__device__ __forceinline__ void activate(float (&y)[4], int activation) {
  switch (activation) {
    case kRelu:
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = y[i] < 0.0f ? 0.0f : y[i];
      break;
    case kSilu:
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] *= __builtin_amdgcn_rcpf(1.0f + exp_of(-y[i]));
      break;
    case kGelu:
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = y[i], t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.44f * 0.70710678f, fabsf(x), 1.0f));
        float p = __builtin_fmaf(0.03561173379f, t, -0.13897401094f);
        p = __builtin_fmaf(p, t, 0.14834374189f);
        p = __builtin_fmaf(p, t, -0.01009032503f);
        p = __builtin_fmaf(p, t, 0.10790611058f);
        p = __builtin_fmaf(p, t, 0.10865677893f);
        p = __builtin_fmaf(p, t, 0.12443558872f);
        p = __builtin_fmaf(p, t, 0.12411047518f);
        const float half = p * t * __builtin_amdgcn_exp2f(-0.72134752f * (x * x));
        y[i] = x * (x < 0.0f ? half : 1.0f - half);
      }
      break;
    case kGeluTanh:  // (1 + tanh z) / 2 = 1 / (1 + exp(-2 z))
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = y[i], z = x * __builtin_fmaf(0.0713548163f, x * x, 1.59576912f);
        y[i] = x * __builtin_amdgcn_rcpf(1.0f + exp_of(-z));
      }
      break;
  }
}

// COUNT neighbouring elements (2 or 4) of a row, `have` of them in it, as binary32
// and back.
template <int COUNT>
__device__ __forceinline__ void load_part(const void *p, int type, int64_t at, int have, float (&v)[4]) {
  if (have >= COUNT) {
    if (type == kF32) {
      __builtin_memcpy(v, (const float *)p + at, 4 * COUNT);
    } else {
      uint16_t h[COUNT];
      __builtin_memcpy(h, (const uint16_t *)p + at, 2 * COUNT);
#pragma unroll
      for (int i = 0; i < COUNT; ++i) v[i] = type == kF16 ? f16_value(h[i]) : bf16_value(h[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < COUNT; ++i)
      v[i] = i >= have ? 0.0f : type == kF32 ? load_value<kF32>(p, at + i) : type == kF16 ? load_value<kF16>(p, at + i) : load_value<kBF16>(p, at + i);
  }
}
template <int COUNT>
__device__ __forceinline__ void store_part(void *p, int type, int64_t at, int have, const float (&v)[4]) {
  if (have >= COUNT) {  // one store at any alignment
    if (type == kF32) {
      __builtin_memcpy((float *)p + at, v, 4 * COUNT);
    } else {
      uint16_t h[COUNT];
#pragma unroll
      for (int i = 0; i < COUNT; ++i) h[i] = type == kF16 ? f16_bits(v[i]) : bf16_bits(v[i]);
      __builtin_memcpy((uint16_t *)p + at, h, 2 * COUNT);
    }
  } else {
#pragma unroll
    for (int i = 0; i < COUNT; ++i)
      if (i < have) {
        if (type == kF32) store_value<kF32>(p, at + i, v[i]);
        else if (type == kF16) store_value<kF16>(p, at + i, v[i]);
        else store_value<kBF16>(p, at + i, v[i]);
      }
  }
}

// The same tile with an activation and the residual stream.  The stream's values
// of a row are asked for before the row above is stored: where the result takes
// the stream's place the compiler may not do so by itself.
template <class S>
__device__ __forceinline__ void store_finished(const MatmulArgs &A, int m, int n, int lane, int4v (&acc)[S::MT][S::NT],
                                               const float (&sa)[S::MT]) {
  float4v sw[S::NT], bias[S::NT] = {};
#pragma unroll
  for (int j = 0; j < S::NT; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int channel = min(n + j * 16 + (lane >> 4) * 4 + i, A.N - 1);
      sw[j][i] = A.w_scale[channel];
      if (A.bias) bias[j][i] = A.bias[channel];
    }
  float stream[2][S::NT][4] = {};
  const auto ask = [&](int i) {
    const int row = m + i * 16 + (lane & 15);
#pragma unroll
    for (int j = 0; j < S::NT; ++j) {
      const int channel = n + j * 16 + (lane >> 4) * 4;
      if (row < A.M && channel < A.N)
        load_part<4>(A.residual, A.out_type, (int64_t)row * A.residual_stride + channel, A.N - channel, stream[i & 1][j]);
    }
  };
  if (A.residual) ask(0);
#pragma unroll
  for (int i = 0; i < S::MT; ++i) {
    if (A.residual && i + 1 < S::MT) ask(i + 1);
    const int row = m + i * 16 + (lane & 15);
#pragma unroll
    for (int j = 0; j < S::NT; ++j) {
      const int channel = n + j * 16 + (lane >> 4) * 4;
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[e] = (float)acc[i][j][e] * sa[i] * sw[j][e];
        if (A.bias) y[e] += bias[j][e];
      }
      activate(y, A.activation);
      if (A.residual) {
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] += stream[i & 1][j][e];
      }
      if (row < A.M && channel < A.N) store_part<4>(A.out, A.out_type, (int64_t)row * A.out_stride + channel, A.N - channel, y);
    }
  }
}

// A gated tile: a lane has the sums of a channel's gate and of its value.
template <class S>
__device__ __forceinline__ void store_gated(const MatmulArgs &A, int m, int n, int lane, int4v (&acc)[S::MT][S::NT],
                                            const float (&sa)[S::MT]) {
  constexpr int PARTS = S::NT == 1 ? 1 : S::NT / 2, COUNT = S::NT == 1 ? 2 : 4;
  float sg[PARTS][4] = {}, sv[PARTS][4] = {}, bg[PARTS][4] = {}, bv[PARTS][4] = {};
#pragma unroll
  for (int j = 0; j < PARTS; ++j)
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      const int64_t channel = min(n + j * 16 + (lane >> 4) * COUNT + i, A.N - 1);
      sg[j][i] = A.w_scale[channel];
      sv[j][i] = A.w_scale[A.N + channel];
      if (A.bias) {
        bg[j][i] = A.bias[channel];
        bv[j][i] = A.bias[A.N + channel];
      }
    }
#pragma unroll
  for (int i = 0; i < S::MT; ++i) {
    const int row = m + i * 16 + (lane & 15);
#pragma unroll
    for (int j = 0; j < PARTS; ++j) {
      const int channel = n + j * 16 + (lane >> 4) * COUNT;
      float gate[4] = {}, value[4] = {};
#pragma unroll
      for (int e = 0; e < COUNT; ++e) {
        gate[e] = (float)acc[i][j][e] * sa[i] * sg[j][e];
        value[e] = (float)(S::NT == 1 ? acc[i][0][(2 + e) & 3] : acc[i][(PARTS + j) % S::NT][e]) * sa[i] * sv[j][e];
        if (A.bias) {
          gate[e] += bg[j][e];
          value[e] += bv[j][e];
        }
      }
      activate(gate, A.activation);
#pragma unroll
      for (int e = 0; e < COUNT; ++e) value[e] *= gate[e];
      if (row < A.M && channel < A.N)
        store_part<COUNT>(A.out, A.out_type, (int64_t)row * A.out_stride + channel, A.N - channel, value);
    }
  }
}

template <class S, Finish FINISH>
__device__ __forceinline__ void finish_tile(const MatmulArgs &A, int m, int n, int lane, int4v (&acc)[S::MT][S::NT],
                                            const float (&sa)[S::MT]) {
  if constexpr (FINISH == kScaled) store_tile<S>(A, m, n, lane, acc, sa);
  else if constexpr (FINISH == kFinished) store_finished<S>(A, m, n, lane, acc, sa);
  else store_gated<S>(A, m, n, lane, acc, sa);
}

// Which operands go from memory to LDS as they are: both where all rows start on
// multiples of 16 bytes, the codes where those rows do and hold whole pieces of
// 16 (fs_linear's and fs_project's own do whatever K is), else none.
enum Direct { kBoth, kCodes, kNone };

template <class S, Direct DIRECT, Finish FINISH>
__global__ __launch_bounds__(S::THREADS) void k_matmul(MatmulArgs A, int tiles_m, int tiles_n) {
  __shared__ __attribute__((aligned(1024))) int8_t lds[S::BYTES];
  // Workgroups go round the eight XCDs in turn: each XCD gets a run of tiles,
  // in groups of eight rows of tiles, so that its L2 serves both operands.
  // (Finished products: an XCD's tiles behind the first A.whole are cut into A.parts
  // along the inner dimension, a block a part.)
  const int total = tiles_m * tiles_n, per = (total + 7) / 8, xcd = blockIdx.x & 7;
  int in_xcd = blockIdx.x >> 3, part = 0, parts = 1;
  if (FINISH != kScaled && in_xcd >= A.whole) {
    parts = A.parts;
    part = (in_xcd - A.whole) % parts;
    in_xcd = A.whole + (in_xcd - A.whole) / parts;
  }
  const int id = xcd * per + in_xcd;
  if (in_xcd >= per || id >= total) return;
  const int group = id / (8 * tiles_n), gm = min(8, tiles_m - group * 8), in = id - group * 8 * tiles_n;
  const int m0 = (group * 8 + in % gm) * S::BM, n0 = in / gm * kChannels<S, FINISH>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wk = wave / S::TILES, wt = wave % S::TILES;
  const int wm = wt / (S::BN / S::WN) * S::WM, wn = wt % (S::BN / S::WN) * S::WN;
  const int each = A.K / S::BK / parts * S::BK, k0 = part * each, K = part == parts - 1 ? A.K - k0 : each;
  const int8_t *const ta = A.a + (int64_t)m0 * A.a_stride + k0, *const tw = A.w + (int64_t)n0 * A.w_stride + k0;
  const int last_a = A.M - 1 - m0, last_w = A.N - 1 - n0;
  // a weight row of the tile, in rows from its first one on
  const auto from_w = [&](int r) {
    const WeightRow row = weight_row<S, FINISH>(r);
    return min(row.channel, last_w) + (row.value ? A.N : 0);
  };
  int4v acc[S::MT][S::NT] = {};
  int done = 0;

  if constexpr (DIRECT == kCodes) {
    // Weights at any alignment go through registers to their slot of the ring,
    // a stage or two ahead, behind the codes of the same stage.  The last stage's
    // weights end in zeros, so whatever codes stand beside them are of no account:
    // places beyond the row take its last piece.  (us a call, so and with
    // both operands through registers: 333 x 1001 x 1999 11.8 and 14.5, 64 x 5001 x
    // 5119 18.2 and 23.3, 3000 x 5001 x 2999 76 and 89.)
    constexpr int AHEAD = S::NS >= 3 && S::MT * S::NT <= 8 ? 2 : 1;
    const int stages = (K + S::BK - 1) / S::BK;
    const uint32_t base = (uint32_t)(size_t)(__attribute__((address_space(3))) int8_t *)lds + wave * 1024;
    Piece rw[AHEAD][S::LW];
    uint32_t row_a[S::LA];
    const int8_t *pw[S::LW];
#pragma unroll
    for (int i = 0; i < S::LA; ++i) row_a[i] = (uint32_t)min(place<S>(i).x, last_a) * (uint32_t)A.a_stride;
#pragma unroll
    for (int i = 0; i < S::LW; ++i) pw[i] = tw + (int64_t)from_w(place<S>(i).x) * A.w_stride;
    const int last_piece = (K - 1) & ~15;
    const auto fetch = [&](int p, int t, int slot) {
#pragma unroll
      for (int i = 0; i < S::LA; ++i)
        load_to_lds(ta, row_a[i] + min(t * S::BK + place<S>(i).y, last_piece), base + slot * S::STAGE + i * S::THREADS * 16);
      const bool over = (t + 1) * S::BK > K;
#pragma unroll
      for (int i = 0; i < S::LW; ++i) rw[p][i].load(pw[i], t * S::BK + place<S>(i).y, K, over);
    };
#pragma unroll
    for (int p = 0; p < AHEAD; ++p)
      if (p < stages) fetch(p, p, p);
    for (int t0 = 0, slot = 0; t0 < stages; t0 += AHEAD) {
#pragma unroll
      for (int p = 0; p < AHEAD; ++p) {
        const int t = t0 + p;
        if (t >= stages) break;
        const bool over = (t + 1) * S::BK > K;
        int8_t *const la = lds + slot * S::STAGE, *const lw = la + S::PART_A;
#pragma unroll
        for (int i = 0; i < S::LW; ++i)
          *(int4v *)(lw + (i * S::THREADS + threadIdx.x) * 16) = rw[p][i].codes(t * S::BK + place<S>(i).y, K, over);
        // the codes of stage t: behind them its weights' loads and a stage's where two are under way
        if (t + 1 < stages) wait_loads<(AHEAD == 2 ? S::LA + 2 * S::LW : S::LW)>();
        else wait_loads<0>();
        __builtin_amdgcn_s_barrier();  // all of stage t is there, and all have read stage t - 1
        asm volatile("" ::: "memory");
        if (t + AHEAD < stages) fetch(p, t + AHEAD, (slot + AHEAD) % S::NS);
        multiply_stage<S>(la, lw, wm, wn, wk, lane, acc);
        slot = slot == S::NS - 1 ? 0 : slot + 1;
      }
    }
    done = K;
  }
  if constexpr (DIRECT == kBoth) {
    const int full = K / S::BK;
    const uint32_t base = (uint32_t)(size_t)(__attribute__((address_space(3))) int8_t *)lds + wave * 1024;
    // a lane's places in a stage, from the tile's first row on (strides fit 32 bits: see matmul_as)
    uint32_t oa[S::LA], ow[S::LW];
#pragma unroll
    for (int i = 0; i < S::LA; ++i) oa[i] = (uint32_t)min(place<S>(i).x, last_a) * (uint32_t)A.a_stride + place<S>(i).y;
#pragma unroll
    for (int i = 0; i < S::LW; ++i) ow[i] = (uint32_t)from_w(place<S>(i).x) * (uint32_t)A.w_stride + place<S>(i).y;
    const auto load = [&](int t, int slot) {
#pragma unroll
      for (int i = 0; i < S::LA; ++i)
        load_to_lds(ta + (int64_t)t * S::BK, oa[i], base + slot * S::STAGE + i * S::THREADS * 16);
#pragma unroll
      for (int i = 0; i < S::LW; ++i)
        load_to_lds(tw + (int64_t)t * S::BK, ow[i], base + slot * S::STAGE + S::PART_A + i * S::THREADS * 16);
    };
    for (int t = 0; t < S::NS - 1 && t < full; ++t) load(t, t);
    for (int t = 0, slot = 0; t < full; ++t, slot = slot == S::NS - 1 ? 0 : slot + 1) {
      const int left = full - 1 - t;
      wait_stage<S::NS, S::LA + S::LW>(left);
      // all wavefronts' loads of stage t are there, and all have read stage t - 1
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (left >= S::NS - 1) load(t + S::NS - 1, slot ? slot - 1 : S::NS - 1);
      multiply_stage<S>(lds + slot * S::STAGE, lds + slot * S::STAGE + S::PART_A, wm, wn, wk, lane, acc);
    }
    done = full * S::BK;
  }
  // Rows at any alignment, or their last part: through registers, AHEAD stages'
  // loads under way (as many as there are registers for).
  if (DIRECT != kCodes && done < K) {
    constexpr int AHEAD = DIRECT == kBoth || S::MT * S::NT > 8 ? 1 : 2;
    Piece ra[AHEAD][S::LA], rw[AHEAD][S::LW];
    const int8_t *pa[S::LA], *pw[S::LW];
#pragma unroll
    for (int i = 0; i < S::LA; ++i) pa[i] = ta + (int64_t)min(place<S>(i).x, last_a) * A.a_stride;
#pragma unroll
    for (int i = 0; i < S::LW; ++i) pw[i] = tw + (int64_t)from_w(place<S>(i).x) * A.w_stride;
    const auto fetch = [&](int p, int k) {
      const bool over = k + S::BK > K;
#pragma unroll
      for (int i = 0; i < S::LA; ++i) ra[p][i].load(pa[i], k + place<S>(i).y, K, over);
#pragma unroll
      for (int i = 0; i < S::LW; ++i) rw[p][i].load(pw[i], k + place<S>(i).y, K, over);
    };
#pragma unroll
    for (int p = 0; p < AHEAD; ++p)
      if (done + p * S::BK < K) fetch(p, done + p * S::BK);
    for (int k0 = done; k0 < K; k0 += AHEAD * S::BK) {
#pragma unroll
      for (int p = 0; p < AHEAD; ++p) {
        const int k = k0 + p * S::BK;
        if (k >= K) break;
        const bool over = k + S::BK > K;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < S::LA; ++i)
          *(int4v *)(lds + (i * S::THREADS + threadIdx.x) * 16) = ra[p][i].codes(k + place<S>(i).y, K, over);
#pragma unroll
        for (int i = 0; i < S::LW; ++i)
          *(int4v *)(lds + S::PART_A + (i * S::THREADS + threadIdx.x) * 16) = rw[p][i].codes(k + place<S>(i).y, K, over);
        __syncthreads();
        if (k + AHEAD * S::BK < K) fetch(p, k + AHEAD * S::BK);
        multiply_stage<S>(lds, lds + S::PART_A, wm, wn, wk, lane, acc);
      }
    }
  }
  const bool mine = join_parts<S>(lds, wk, wave, lane, acc);
  if constexpr (FINISH != kScaled)
    if (parts > 1 && !join_blocks<S>(A, xcd * (per - A.whole) + in_xcd - A.whole, part, parts, mine, wt, lane, acc)) return;
  if (!mine) return;
  float sa[S::MT];
#pragma unroll
  for (int i = 0; i < S::MT; ++i) sa[i] = A.a_scale[min(m0 + wm + i * 16 + (lane & 15), A.M - 1)];
  finish_tile<S, FINISH>(A, m0 + wm, n0 + (FINISH == kGated ? wn / 2 : wn), lane, acc, sa);
}

// ------------------------------------------------- few rows, in one launch --
// A projection of up to four rows: every block makes the codes of all of them
// itself, so that no kernel has to end before another starts.  The rows go to
// LDS as they are, behind them the first stages of weights are under way while
// the largest values are found and the codes made.  A last stage that passes
// K ends in codes of zero, and its weights are the row's last ones again.
constexpr int kFewRows = 4, kFewThreads = 512, kFewBytes = 152 << 10;

// Codes of the rows in LDS (`raw`, rows `raw_pitch` bytes apart) and their
// scales.  The block's wavefronts share out the rows.
// `gain`: in LDS, or NULL; NORMED as in k_quantize_rows.
template <class S, int XTYPE, bool NORMED>
__device__ __forceinline__ void codes_in_lds(const int8_t *raw, int raw_pitch, int8_t *codes, int pitch, float *scales,
                                             uint32_t *most_of, int M, int K, int wave, int lane, const float *gain,
                                             float eps, Squares *squares) {
  const int each = S::WAVES / (M == 1 ? 1 : M == 2 ? 2 : 4);  // wavefronts of a row
  const int row = wave / each, first = (wave % each * 64 + lane) * 8, step = each * 512;
  const int8_t *const from = raw + row * raw_pitch;
  uint32_t most = 0;
  Squares sum = {0.0f, 0.0f};
  constexpr int HELD = NORMED ? 2 : 1;
  float normed[HELD][8] = {};  // of a row of two steps or less, between the passes
  const auto norm = [&](int c, float(&v)[8]) {
    float g[8];
    load8<XTYPE>(from, c, true, v);
    gain8(gain, c, K, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sum.add(v[i]);
      v[i] *= g[i];
      most = max(most, magnitude(v[i]));
    }
  };
  if (row < M) {
    if constexpr (NORMED) {
      if (K <= HELD * step) {
#pragma unroll
        for (int j = 0; j < HELD; ++j)
          if (first + j * step < K) norm(first + j * step, normed[j]);
      } else {
        for (int c = first; c < K; c += step) norm(c, normed[0]);
      }
      sum.join_lanes();
    } else if constexpr (XTYPE == kF32) {
      for (int c = first; c < K; c += step) {
        float v[8];
        load8<XTYPE>(from, c, true, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[i]));
      }
    } else {  // without the sign the types' words are in the values' order
      using short2 = uint16_t __attribute__((ext_vector_type(2)));
      short2 two = {0, 0};
      for (int c = first; c < K; c += step) {
        const int4v raw = *(const int4v *)(from + 2 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) two = __builtin_elementwise_max(two, __builtin_bit_cast(short2, raw[i] & 0x7fff7fff));
      }
      most = magnitude(value16<XTYPE>(max(two.x, two.y)));
    }
  }
  most = wave_max(most);
  if (lane == 0) most_of[wave] = most;
  if constexpr (NORMED) {
    if (lane == 0) squares[wave] = sum;
  }
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // LDS only: the weights' loads stay under way
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  for (int i = 0; i < each; ++i) most = max(most, most_of[row * each + i]);
  const float a = __uint_as_float(most);
  const bool zero = a < kTiny;
  const float inverse = zero ? 0.0f : 127.0f / a;
  if (NORMED && row < M && K <= HELD * step) {
#pragma unroll
    for (int j = 0; j < HELD + 1; ++j) {  // a row's codes end in zeros, less than a step of them
      const int c = first + j * step;
      if (c < pitch) *(int2 *)(codes + row * pitch + c) = codes8(normed[j < HELD ? j : 0], j < HELD && c < K ? inverse : 0.0f);
    }
  } else if (row < M) {
    for (int c = first; c < pitch; c += step) {
      float v[8] = {};
      if (c < K) load8<XTYPE>(from, c, true, v);
      if constexpr (NORMED) {
        float g[8];
        if (c < K) {
          gain8(gain, c, K, g);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] *= g[i];
        }
      }
      *(int2 *)(codes + row * pitch + c) = codes8(v, c < K ? inverse : 0.0f);
    }
  }
  if (row < M) {
    if (first == 0) {
      if constexpr (NORMED) {
        sum = squares[row * each];
        for (int i = 1; i < each; ++i) sum.add(squares[row * each + i]);
        scales[row] = zero ? 0.0f : a * sum.factor(K, eps) / 127.0f;
      } else {
        scales[row] = zero ? 0.0f : a / 127.0f;
      }
    }
  }
  asm volatile("" ::: "memory");
}

template <class S, Finish FINISH, bool NORMED>
__global__ __launch_bounds__(S::THREADS) void k_linear_few(QuantizeArgs X, MatmulArgs A, int tiles_n) {
  extern __shared__ __attribute__((aligned(1024))) int8_t few_lds[];
  __shared__ float scales[kFewRows];
  __shared__ uint32_t most_of[S::WAVES];
  __shared__ Squares squares[NORMED ? S::WAVES : 1];
  constexpr int STAGE = S::BN * S::BK;
  const int per = (tiles_n + 7) / 8, id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || id >= tiles_n) return;
  const int n0 = id * kChannels<S, FINISH>, stages = (A.K + S::BK - 1) / S::BK;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wk = wave / S::TILES, wn = wave % S::TILES * S::WN;
  const int x_bytes = A.K * (X.type == kF32 ? 4 : 2), x_loads = (x_bytes + S::THREADS * 16 - 1) / (S::THREADS * 16);
  const int raw_pitch = x_loads * S::THREADS * 16, pitch = stages * S::BK + 64;
  int8_t *const raw = few_lds + S::NS * STAGE, *const codes = raw + A.M * raw_pitch;
  int8_t *const gain = codes + A.M * pitch;  // behind the codes, whose length is a multiple of 64
  const uint32_t base = (uint32_t)(size_t)(__attribute__((address_space(3))) int8_t *)few_lds + wave * 1024;

  for (int m = 0; m < A.M; ++m)
    for (int i = 0; i < x_loads; ++i)
      load_to_lds((const int8_t *)X.x + m * X.x_stride * (X.type == kF32 ? 4 : 2),
                  (uint32_t)min((i * S::THREADS + (int)threadIdx.x) * 16, x_bytes - 16),
                  base + S::NS * STAGE + m * raw_pitch + i * S::THREADS * 16);
  if (NORMED && X.gain) {
    const int gain_bytes = A.K * 4, loads = (gain_bytes + S::THREADS * 16 - 1) / (S::THREADS * 16);
    for (int i = 0; i < loads; ++i)
      load_to_lds((const int8_t *)X.gain, (uint32_t)min((i * S::THREADS + (int)threadIdx.x) * 16, gain_bytes - 16),
                  base + (uint32_t)(gain - few_lds) + i * S::THREADS * 16);
  }
  const int8_t *const tw = A.w + (int64_t)n0 * A.w_stride;
  uint32_t row_at[S::LW];
  int in_row[S::LW];
#pragma unroll
  for (int i = 0; i < S::LW; ++i) {
    const int2 at = place<S>(i);
    const WeightRow row = weight_row<S, FINISH>(at.x);
    row_at[i] = (uint32_t)(min(row.channel, A.N - 1 - n0) + (row.value ? A.N : 0)) * (uint32_t)A.w_stride;
    in_row[i] = at.y;
  }
  const auto load = [&](int t, int slot) {
#pragma unroll
    for (int i = 0; i < S::LW; ++i)
      load_to_lds(tw, row_at[i] + min(t * S::BK + in_row[i], A.K - 16), base + slot * STAGE + i * S::THREADS * 16);
  };
  for (int t = 0; t < S::NS - 1 && t < stages; ++t) load(t, t);
  if (stages >= S::NS - 1) wait_loads<(S::NS - 1) * S::LW>();
  else wait_loads<0>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  const float *const gains = NORMED && X.gain ? (const float *)gain : nullptr;
  if (X.type == kF32) codes_in_lds<S, kF32, NORMED>(raw, raw_pitch, codes, pitch, scales, most_of, A.M, A.K, wave, lane, gains, X.eps, squares);
  else if (X.type == kF16) codes_in_lds<S, kF16, NORMED>(raw, raw_pitch, codes, pitch, scales, most_of, A.M, A.K, wave, lane, gains, X.eps, squares);
  else codes_in_lds<S, kBF16, NORMED>(raw, raw_pitch, codes, pitch, scales, most_of, A.M, A.K, wave, lane, gains, X.eps, squares);

  int4v acc[1][S::NT] = {};
  const int r = lane & 15;
  const int8_t *const own = codes + min(r, A.M - 1) * pitch;  // the rows beyond M are no one's
  constexpr int STEPS = S::BK / 64 / S::WK;
  for (int t = 0, slot = 0; t < stages; ++t, slot = slot == S::NS - 1 ? 0 : slot + 1) {
    const int left = stages - 1 - t;
    wait_stage<S::NS, S::LW>(left);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (left >= S::NS - 1) load(t + S::NS - 1, slot ? slot - 1 : S::NS - 1);
    const int8_t *const lw = few_lds + slot * STAGE;
#pragma unroll
    for (int kk = 0; kk < STEPS; ++kk) {
      const int chunk = (wk * STEPS + kk) * 4 + (lane >> 4);
      const int4v fa = *(const int4v *)(own + t * S::BK + chunk * 16);
#pragma unroll
      for (int j = 0; j < S::NT; ++j) {
        const int4v fw = *(const int4v *)(lw + (wn + j * 16 + r) * S::BK + (chunk ^ turn<S::BK>(r)) * 16);
        acc[0][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw, fa, acc[0][j], 0, 0, 0);
      }
    }
  }
  if (!join_parts<S>(few_lds, wk, wave, lane, acc)) return;
  const float sa[1] = {scales[min(r, A.M - 1)]};
  finish_tile<S, FINISH>(A, 0, n0 + (FINISH == kGated ? wn / 2 : wn), lane, acc, sa);
}

template <int TYPE, int THREADS, int HELD, bool NORMED>
hipError_t quantize_as(const QuantizeArgs &A, hipStream_t s) {
  constexpr int64_t MOST = kMostBlocks / 2;  // blocks have up to 1024 threads
  for (int64_t r = 0; r < A.rows; r += MOST) {
    QuantizeArgs part = A;
    part.x = (const uint8_t *)A.x + r * A.x_stride * (TYPE == kF32 ? 4 : 2);
    part.codes = A.codes + r * A.code_stride;
    part.scale = A.scale + r;
    part.rows = (int32_t)std::min(MOST, A.rows - r);
    k_quantize_rows<TYPE, THREADS, HELD, NORMED><<<part.rows, THREADS, 0, s>>>(part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int TYPE, bool NORMED>
hipError_t quantize_of(const QuantizeArgs &A, hipStream_t s) {
  // few rows: all of a CU's wavefronts on one; many: smaller blocks
  if (A.rows <= 256 && A.cols <= 8192) return quantize_as<TYPE, 1024, 1, NORMED>(A, s);
  if (A.rows <= 256 && A.cols <= 3 * 8192) return quantize_as<TYPE, 1024, 3, NORMED>(A, s);
  if (A.cols <= 4 * 2048) return quantize_as<TYPE, 256, 4, NORMED>(A, s);
  if (A.cols <= 10 * 2048) return quantize_as<TYPE, 256, 10, NORMED>(A, s);
  return quantize_as<TYPE, 1024, 0, NORMED>(A, s);
}

template <int TYPE, Finish FINISH, int BM, int BN, int WM, int WN, int BK, int WK, int NS>
hipError_t matmul_as(const MatmulArgs &A, hipStream_t s) {
  using S = Shape<TYPE, BM, BN, WM, WN, BK, WK, NS>;
  const int tm = (A.M - 1) / BM + 1, tn = (A.N - 1) / kChannels<S, FINISH> + 1;
  // see matmul_fits and choose
  const int grid = FINISH == kScaled ? (tm * tn + 7) / 8 * 8 : 8 * (A.whole + ((tm * tn + 7) / 8 - A.whole) * A.parts);
  const auto whole = [](const int8_t *p, int64_t stride) { return (((uintptr_t)p | (uintptr_t)stride) & 15) == 0 && stride <= 1 << 23; };
  // (both rows of a gated channel: in 32 bits from the tile's first on)
  const bool a = whole(A.a, A.a_stride), w = whole(A.w, A.w_stride) && (FINISH != kGated || A.N * A.w_stride <= (int64_t)1 << 31);
  if (a && w) k_matmul<S, kBoth, FINISH><<<grid, S::THREADS, 0, s>>>(A, tm, tn);
  else if (FINISH != kScaled || (a && (A.a_padded || A.K % 16 == 0))) k_matmul<S, kCodes, FINISH><<<grid, S::THREADS, 0, s>>>(A, tm, tn);
  else if constexpr (FINISH == kScaled) k_matmul<S, kNone, FINISH><<<grid, S::THREADS, 0, s>>>(A, tm, tn);
  return hipGetLastError();
}

// The tile whose rounds over the 256 CUs take least: a round's time is about
// 1.5 us and, for each 5120 inner elements, what is measured with the tile at
// one block a CU.  (K = 5120, us of the product alone, one call after another:
// 64 tokens x 5120 channels 9.0 with tiles of 64 x 32, 12.1 with 32 x 32, 11.1
// with 64 x 64; 64 x 896 4.3 with 16 x 16 and 6.2 with 32 x 32; 128 x 5120 11.3
// with 64 x 64, 15.9 with 64 x 32; 2048 x 5120 70 with 128 x 64 and with 256 x
// 256; 8192 x 20480 743 with 256 x 256, 847 with 256 x 128.)
struct Tile {
  int bm, bn;
  double us;
};
constexpr Tile kTiles[] = {{16, 16, 2.4},  {16, 32, 5.5},   {32, 32, 6.1},    {64, 32, 8.1},   {64, 64, 11.1},
                           {128, 64, 13.0}, {128, 128, 25.0}, {256, 128, 43.5}, {256, 256, 78.0}};

int best_tile(int32_t M, int32_t N, int32_t K) {
  int best = 0;
  double least = 0.0;
  for (int i = 0; i < (int)(sizeof(kTiles) / sizeof(kTiles[0])); ++i) {
    const Tile &t = kTiles[i];
    const int64_t tiles = ((int64_t)(M + (int64_t)t.bm - 1) / t.bm) * ((N + (int64_t)t.bn - 1) / t.bn);
    const double time = (double)((tiles + 255) / 256) * (1.5 + t.us * K / 5120.0);
    if (i == 0 || time < least) {
      best = i;
      least = time;
    }
  }
  return best;
}

// The same for products that may be cut along the inner dimension: tiles of all 256
// CUs whole, and those of the last round, if they are no more than half of them,
// in as many parts as there are CUs for.  A part costs its writing and, but the
// last's, its reading, at 4 TB/s, and what waits for them 3 us.  (N: rows of w.
// us a call, with the quantisation, weights from memory, best uncut and cut: 64 x 5120 x
// 20480 44 and 36, 64 x (2 x 20480) x 5120 58.9 and 58.0, 8192 x 5120 x 20480 872 and 852.
// The tiles' times are those of weights that start on 16 bytes; others take up to twice
// as long: 333 x 1001 x 1999 4.7 us expected, 8.9 measured.)
constexpr int64_t kMostParts = 256, kLeastPart = 1024;  // a block a CU, inner elements of each

struct Choice {
  int tile, parts;
  int64_t whole, rest;  // tiles of an XCD that are whole, and cut into parts

  int64_t slots() const { return parts > 1 ? 8 * rest : 0; }
  int64_t bytes() const { return slots() * parts * kTiles[tile].bm * kTiles[tile].bn * 4; }
};

Choice choose(int32_t M, int32_t N, int32_t K) {
  Choice best{};
  double least = 0.0;
  for (int i = 0; i < (int)(sizeof(kTiles) / sizeof(kTiles[0])); ++i) {
    const Tile &t = kTiles[i];
    const int64_t tiles = ((int64_t)(M + (int64_t)t.bm - 1) / t.bm) * ((N + (int64_t)t.bn - 1) / t.bn);
    const int64_t per = (tiles + 7) / 8, rest = per % 32;
    const double one = t.us * K / 5120.0, time = (double)((per + 31) / 32) * (1.5 + one);
    if (i == 0 || time < least) {
      best = {i, 1, per, 0};
      least = time;
    }
    const int parts = rest ? (int)std::min<int64_t>(kMostParts / 8 / rest, K / kLeastPart) : 1;
    if (parts < 2) continue;
    const double moved = 8.0 * rest * (2 * parts - 1) * t.bm * t.bn * 4 / 4e6;
    const double cut = (double)(per / 32) * (1.5 + one) + 1.5 + one / parts + 3.0 + moved;
    if (cut < least) {
      best = {i, parts, per - rest, rest};
      least = cut;
    }
  }
  return best;
}

template <int TYPE, Finish FINISH>
hipError_t matmul_of(const MatmulArgs &A, hipStream_t s) {
  switch (FINISH == kScaled ? best_tile(A.M, A.N, A.K) : A.tile) {
    case 0: return matmul_as<TYPE, FINISH, 16, 16, 16, 16, 512, 8, 4>(A, s);
    case 1: return matmul_as<TYPE, FINISH, 16, 32, 16, 16, 512, 4, 3>(A, s);
    case 2: return matmul_as<TYPE, FINISH, 32, 32, 16, 16, 512, 2, 4>(A, s);
    case 3: return matmul_as<TYPE, FINISH, 64, 32, 32, 16, 512, 2, 3>(A, s);
    case 4: return matmul_as<TYPE, FINISH, 64, 64, 32, 32, 256, 2, 4>(A, s);
    case 5: return matmul_as<TYPE, FINISH, 128, 64, 32, 32, 128, 1, 3>(A, s);
    case 6: return matmul_as<TYPE, FINISH, 128, 128, 32, 64, 128, 1, 3>(A, s);
    case 7: return matmul_as<TYPE, FINISH, 256, 128, 64, 64, 128, 1, 3>(A, s);
    default: return matmul_as<TYPE, FINISH, 256, 256, 128, 64, 128, 1, 2>(A, s);
  }
}

template <int TYPE, Finish FINISH, bool NORMED, int BN, int WK, int NS>
hipError_t few_as(const QuantizeArgs &X, const MatmulArgs &A, int64_t rows_bytes, hipStream_t s) {
  using S = Shape<TYPE, 16, BN, 16, 16, 512, WK, NS>;
  constexpr int RING = S::NS * S::BN * S::BK;
  static_assert(RING >= S::WAVES * S::NT * 1024, "the parts' sums fit the ring");
  static_assert(S::THREADS == kFewThreads, "whole loads of a row");
  // more than 64 KB of LDS asked for at the launch
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_linear_few<S, FINISH, NORMED>), hipFuncAttributeMaxDynamicSharedMemorySize, kFewBytes);
  if (e != hipSuccess) return e;
  const int tiles = (A.N - 1) / kChannels<S, FINISH> + 1;
  k_linear_few<S, FINISH, NORMED><<<(tiles + 7) / 8 * 8, S::THREADS, (size_t)(RING + rows_bytes), s>>>(X, A, tiles);
  return hipGetLastError();
}

// Where one launch is faster than two: a block a CU or less, or a single row
// and two blocks a CU.  (bfloat16, eight sets of weights in turn, us of one
// launch and of two: 1 x 7168 x 5120 8.9 and 11.6, 4 rows 10.4 and 11.6; 1 x 896
// x 5120 5.3 and 7.3; 1 x 5120 x 640 4.1 and 7.3; 1 x 5120 x 20480 23.5 and 28.6;
// 1 x 10240 x 5120 12.9 and 16.2; 4 x 10240 x 5120 18.9 and 16.2, where every CU
// makes the codes twice.)
template <int TYPE, Finish FINISH, bool NORMED>
bool few_of(const QuantizeArgs &X, const MatmulArgs &A, hipStream_t s, hipError_t *e) {
  const int64_t size = X.type == kF32 ? 4 : 2, load = kFewThreads * 16, rows = FINISH == kGated ? 2 * (int64_t)A.N : A.N;
  const int64_t gain = NORMED && X.gain ? (A.K * 4 + load - 1) / load * load : 0;
  const int64_t bytes = A.M * ((A.K * size + load - 1) / load * load + (A.K + 511) / 512 * 512 + 64) + gain;
  if (rows <= 256 * 16 && 6 * 8192 + bytes <= kFewBytes) *e = few_as<TYPE, FINISH, NORMED, 16, 8, 6>(X, A, bytes, s);
  else if (rows <= 256 * 32 && 4 * 16384 + bytes <= kFewBytes) *e = few_as<TYPE, FINISH, NORMED, 32, 4, 4>(X, A, bytes, s);
  else if (A.M == 1 && 3 * 16384 + bytes <= 80 << 10 && rows <= kMostBlocks * 32) *e = few_as<TYPE, FINISH, NORMED, 32, 4, 3>(X, A, bytes, s);
  else return false;
  return true;
}

// Whether the call is one of few rows at all: loads of 16 bytes, of a row's own.
bool few_rows(const QuantizeArgs &X, const MatmulArgs &A) {
  const int64_t size = X.type == kF32 ? 4 : 2;
  if (A.M > kFewRows || A.K < 16 || A.K % 16 || A.w_stride > (1 << 23)) return false;
  return !(((uintptr_t)X.x | (uintptr_t)(A.M > 1 ? X.x_stride * size : 0) | (uintptr_t)A.w | (uintptr_t)A.w_stride | (uintptr_t)X.gain) & 15);
}

}  // namespace
}  // namespace fs
