// fs_linear.hip -- projections in 8-bit integers: rows of activations to
// codes with a scale a row, and the product of codes with weights that have a
// scale an output channel.
//
// y[m][n] = (sum_k a[m][k] w[n][k]) * a_scale[m] * w_scale[n] + bias[n].
// The sum is exact in 32-bit integers whatever the order, so tiles, splits
// and instructions are free to choose and every variant gives the same bits.
//
// In all variants the weights are the instruction's first operand, so a
// lane's four results are neighbouring channels of one token.
#include <algorithm>

#include "fs_serving.h"

namespace fs {
namespace {

// The largest |x| of a block's values by their bit patterns: a NaN is larger
// than an infinity, so neither is lost in the maximum.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

template <int THREADS>
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t *lds) {
  for (int o = 32; o; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
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
  } else {
    for (int i = 0; i < 8; ++i) v[i] = i < cols - c ? load_value<TYPE>(x, row + c + i) : 0.0f;
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

// One block a row, the row in registers: HELD groups of 8 elements a thread.
// HELD = 0: a row too long for that is read twice (the second time from L2).
template <int TYPE, int THREADS, int HELD>
__global__ __launch_bounds__(THREADS) void k_quantize_rows(QuantizeArgs A) {
  __shared__ uint32_t lds[THREADS / 64];
  const int64_t row = blockIdx.x, at = row * A.x_stride;
  const int own = threadIdx.x * 8, step = THREADS * 8;
  const bool whole = (((uintptr_t)A.x | (uintptr_t)(A.x_stride * 2)) & 15) == 0;
  float v[HELD ? HELD : 1][8];
  uint32_t most = 0;
  if constexpr (HELD > 0) {
#pragma unroll
    for (int j = 0; j < HELD; ++j) load8_of<TYPE>(A.x, at, min(own + j * step, A.cols), A.cols, whole, v[j]);
#pragma unroll
    for (int j = 0; j < HELD; ++j)
      for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[j][i]));
  } else {
    for (int64_t c = own; c < A.cols; c += step) {
      load8_of<TYPE>(A.x, at, (int)c, A.cols, whole, v[0]);
      for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[0][i]));
    }
  }
  const float a = __uint_as_float(block_max<THREADS>(most, lds));
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
      store_codes8(out, (int)c, A.cols, v[0], inverse);
    }
  }
  if (threadIdx.x == 0) A.scale[row] = zero ? 0.0f : a / 127.0f;
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

// Which operands go from memory to LDS as they are: both where all rows start on
// multiples of 16 bytes, the codes where those rows do and hold whole pieces of
// 16 (fs_linear's own do whatever K is), else none.
enum Direct { kBoth, kCodes, kNone };

template <class S, Direct DIRECT>
__global__ __launch_bounds__(S::THREADS) void k_matmul(MatmulArgs A, int tiles_m, int tiles_n) {
  __shared__ __attribute__((aligned(1024))) int8_t lds[S::BYTES];
  // Workgroups go round the eight XCDs in turn: each XCD gets a run of tiles,
  // in groups of eight rows of tiles, so that its L2 serves both operands.
  const int total = tiles_m * tiles_n, per = (total + 7) / 8;
  const int id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || id >= total) return;
  const int group = id / (8 * tiles_n), gm = min(8, tiles_m - group * 8), in = id - group * 8 * tiles_n;
  const int m0 = (group * 8 + in % gm) * S::BM, n0 = in / gm * S::BN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wk = wave / S::TILES, wt = wave % S::TILES;
  const int wm = wt / (S::BN / S::WN) * S::WM, wn = wt % (S::BN / S::WN) * S::WN;
  const int8_t *const ta = A.a + (int64_t)m0 * A.a_stride, *const tw = A.w + (int64_t)n0 * A.w_stride;
  const int last_a = A.M - 1 - m0, last_w = A.N - 1 - n0;
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
    const int stages = (A.K + S::BK - 1) / S::BK;
    const uint32_t base = (uint32_t)(size_t)(__attribute__((address_space(3))) int8_t *)lds + wave * 1024;
    Piece rw[AHEAD][S::LW];
    uint32_t row_a[S::LA];
    const int8_t *pw[S::LW];
#pragma unroll
    for (int i = 0; i < S::LA; ++i) row_a[i] = (uint32_t)min(place<S>(i).x, last_a) * (uint32_t)A.a_stride;
#pragma unroll
    for (int i = 0; i < S::LW; ++i) pw[i] = tw + (int64_t)min(place<S>(i).x, last_w) * A.w_stride;
    const int last_piece = (A.K - 1) & ~15;
    const auto fetch = [&](int p, int t, int slot) {
#pragma unroll
      for (int i = 0; i < S::LA; ++i)
        load_to_lds(ta, row_a[i] + min(t * S::BK + place<S>(i).y, last_piece), base + slot * S::STAGE + i * S::THREADS * 16);
      const bool over = (t + 1) * S::BK > A.K;
#pragma unroll
      for (int i = 0; i < S::LW; ++i) rw[p][i].load(pw[i], t * S::BK + place<S>(i).y, A.K, over);
    };
#pragma unroll
    for (int p = 0; p < AHEAD; ++p)
      if (p < stages) fetch(p, p, p);
    for (int t0 = 0, slot = 0; t0 < stages; t0 += AHEAD) {
#pragma unroll
      for (int p = 0; p < AHEAD; ++p) {
        const int t = t0 + p;
        if (t >= stages) break;
        const bool over = (t + 1) * S::BK > A.K;
        int8_t *const la = lds + slot * S::STAGE, *const lw = la + S::PART_A;
#pragma unroll
        for (int i = 0; i < S::LW; ++i)
          *(int4v *)(lw + (i * S::THREADS + threadIdx.x) * 16) = rw[p][i].codes(t * S::BK + place<S>(i).y, A.K, over);
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
    done = A.K;
  }
  if constexpr (DIRECT == kBoth) {
    const int full = A.K / S::BK;
    const uint32_t base = (uint32_t)(size_t)(__attribute__((address_space(3))) int8_t *)lds + wave * 1024;
    // a lane's places in a stage, from the tile's first row on (strides fit 32 bits: see matmul_as)
    uint32_t oa[S::LA], ow[S::LW];
#pragma unroll
    for (int i = 0; i < S::LA; ++i) oa[i] = (uint32_t)min(place<S>(i).x, last_a) * (uint32_t)A.a_stride + place<S>(i).y;
#pragma unroll
    for (int i = 0; i < S::LW; ++i) ow[i] = (uint32_t)min(place<S>(i).x, last_w) * (uint32_t)A.w_stride + place<S>(i).y;
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
  if (DIRECT != kCodes && done < A.K) {
    constexpr int AHEAD = DIRECT == kBoth || S::MT * S::NT > 8 ? 1 : 2;
    Piece ra[AHEAD][S::LA], rw[AHEAD][S::LW];
    const int8_t *pa[S::LA], *pw[S::LW];
#pragma unroll
    for (int i = 0; i < S::LA; ++i) pa[i] = ta + (int64_t)min(place<S>(i).x, last_a) * A.a_stride;
#pragma unroll
    for (int i = 0; i < S::LW; ++i) pw[i] = tw + (int64_t)min(place<S>(i).x, last_w) * A.w_stride;
    const auto fetch = [&](int p, int k) {
      const bool over = k + S::BK > A.K;
#pragma unroll
      for (int i = 0; i < S::LA; ++i) ra[p][i].load(pa[i], k + place<S>(i).y, A.K, over);
#pragma unroll
      for (int i = 0; i < S::LW; ++i) rw[p][i].load(pw[i], k + place<S>(i).y, A.K, over);
    };
#pragma unroll
    for (int p = 0; p < AHEAD; ++p)
      if (done + p * S::BK < A.K) fetch(p, done + p * S::BK);
    for (int k0 = done; k0 < A.K; k0 += AHEAD * S::BK) {
#pragma unroll
      for (int p = 0; p < AHEAD; ++p) {
        const int k = k0 + p * S::BK;
        if (k >= A.K) break;
        const bool over = k + S::BK > A.K;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < S::LA; ++i)
          *(int4v *)(lds + (i * S::THREADS + threadIdx.x) * 16) = ra[p][i].codes(k + place<S>(i).y, A.K, over);
#pragma unroll
        for (int i = 0; i < S::LW; ++i)
          *(int4v *)(lds + S::PART_A + (i * S::THREADS + threadIdx.x) * 16) = rw[p][i].codes(k + place<S>(i).y, A.K, over);
        __syncthreads();
        if (k + AHEAD * S::BK < A.K) fetch(p, k + AHEAD * S::BK);
        multiply_stage<S>(lds, lds + S::PART_A, wm, wn, wk, lane, acc);
      }
    }
  }
  if (!join_parts<S>(lds, wk, wave, lane, acc)) return;
  float sa[S::MT];
#pragma unroll
  for (int i = 0; i < S::MT; ++i) sa[i] = A.a_scale[min(m0 + wm + i * 16 + (lane & 15), A.M - 1)];
  store_tile<S>(A, m0 + wm, n0 + wn, lane, acc, sa);
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
template <class S, int XTYPE>
__device__ __forceinline__ void codes_in_lds(const int8_t *raw, int raw_pitch, int8_t *codes, int pitch, float *scales,
                                             uint32_t *most_of, int M, int K, int wave, int lane) {
  const int each = S::WAVES / (M == 1 ? 1 : M == 2 ? 2 : 4);  // wavefronts of a row
  const int row = wave / each, first = (wave % each * 64 + lane) * 8, step = each * 512;
  const int8_t *const from = raw + row * raw_pitch;
  uint32_t most = 0;
  if (row < M) {
    if constexpr (XTYPE == kF32) {
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
  for (int o = 32; o; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
  if (lane == 0) most_of[wave] = most;
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // LDS only: the weights' loads stay under way
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  for (int i = 0; i < each; ++i) most = max(most, most_of[row * each + i]);
  const float a = __uint_as_float(most);
  const bool zero = a < kTiny;
  const float inverse = zero ? 0.0f : 127.0f / a;
  if (row < M) {
    for (int c = first; c < pitch; c += step) {
      float v[8] = {};
      if (c < K) load8<XTYPE>(from, c, true, v);
      *(int2 *)(codes + row * pitch + c) = codes8(v, c < K ? inverse : 0.0f);
    }
    if (first == 0) scales[row] = zero ? 0.0f : a / 127.0f;
  }
  asm volatile("" ::: "memory");
}

template <class S>
__global__ __launch_bounds__(S::THREADS) void k_linear_few(QuantizeArgs X, MatmulArgs A, int tiles_n) {
  extern __shared__ __attribute__((aligned(1024))) int8_t few_lds[];
  __shared__ float scales[kFewRows];
  __shared__ uint32_t most_of[S::WAVES];
  constexpr int STAGE = S::BN * S::BK;
  const int per = (tiles_n + 7) / 8, id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || id >= tiles_n) return;
  const int n0 = id * S::BN, stages = (A.K + S::BK - 1) / S::BK;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wk = wave / S::TILES, wn = wave % S::TILES * S::WN;
  const int x_bytes = A.K * (X.type == kF32 ? 4 : 2), x_loads = (x_bytes + S::THREADS * 16 - 1) / (S::THREADS * 16);
  const int raw_pitch = x_loads * S::THREADS * 16, pitch = stages * S::BK + 64;
  int8_t *const raw = few_lds + S::NS * STAGE, *const codes = raw + A.M * raw_pitch;
  const uint32_t base = (uint32_t)(size_t)(__attribute__((address_space(3))) int8_t *)few_lds + wave * 1024;

  for (int m = 0; m < A.M; ++m)
    for (int i = 0; i < x_loads; ++i)
      load_to_lds((const int8_t *)X.x + m * X.x_stride * (X.type == kF32 ? 4 : 2),
                  (uint32_t)min((i * S::THREADS + (int)threadIdx.x) * 16, x_bytes - 16),
                  base + S::NS * STAGE + m * raw_pitch + i * S::THREADS * 16);
  const int8_t *const tw = A.w + (int64_t)n0 * A.w_stride;
  uint32_t row_at[S::LW];
  int in_row[S::LW];
#pragma unroll
  for (int i = 0; i < S::LW; ++i) {
    const int2 at = place<S>(i);
    row_at[i] = (uint32_t)min(at.x, A.N - 1 - n0) * (uint32_t)A.w_stride;
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
  if (X.type == kF32) codes_in_lds<S, kF32>(raw, raw_pitch, codes, pitch, scales, most_of, A.M, A.K, wave, lane);
  else if (X.type == kF16) codes_in_lds<S, kF16>(raw, raw_pitch, codes, pitch, scales, most_of, A.M, A.K, wave, lane);
  else codes_in_lds<S, kBF16>(raw, raw_pitch, codes, pitch, scales, most_of, A.M, A.K, wave, lane);

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
  store_tile<S>(A, 0, n0 + wn, lane, acc, sa);
}

template <int TYPE, int THREADS, int HELD>
hipError_t quantize_as(const QuantizeArgs &A, hipStream_t s) {
  constexpr int64_t MOST = kMostBlocks / 2;  // blocks have up to 1024 threads
  for (int64_t r = 0; r < A.rows; r += MOST) {
    QuantizeArgs part = A;
    part.x = (const uint8_t *)A.x + r * A.x_stride * (TYPE == kF32 ? 4 : 2);
    part.codes = A.codes + r * A.code_stride;
    part.scale = A.scale + r;
    part.rows = (int32_t)std::min(MOST, A.rows - r);
    k_quantize_rows<TYPE, THREADS, HELD><<<part.rows, THREADS, 0, s>>>(part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int TYPE>
hipError_t quantize_of(const QuantizeArgs &A, hipStream_t s) {
  // few rows: all of a CU's wavefronts on one; many: smaller blocks
  if (A.rows <= 256 && A.cols <= 3 * 8192) return quantize_as<TYPE, 1024, 3>(A, s);
  if (A.cols <= 4 * 2048) return quantize_as<TYPE, 256, 4>(A, s);
  if (A.cols <= 10 * 2048) return quantize_as<TYPE, 256, 10>(A, s);
  return quantize_as<TYPE, 1024, 0>(A, s);
}

template <int TYPE, int BM, int BN, int WM, int WN, int BK, int WK, int NS>
hipError_t matmul_as(const MatmulArgs &A, hipStream_t s) {
  using S = Shape<TYPE, BM, BN, WM, WN, BK, WK, NS>;
  const int tm = (A.M - 1) / BM + 1, tn = (A.N - 1) / BN + 1;
  const int grid = (tm * tn + 7) / 8 * 8;  // see matmul_fits
  const auto whole = [](const int8_t *p, int64_t stride) { return (((uintptr_t)p | (uintptr_t)stride) & 15) == 0 && stride <= 1 << 23; };
  const bool a = whole(A.a, A.a_stride), w = whole(A.w, A.w_stride);
  if (a && w) k_matmul<S, kBoth><<<grid, S::THREADS, 0, s>>>(A, tm, tn);
  else if (a && (A.a_padded || A.K % 16 == 0)) k_matmul<S, kCodes><<<grid, S::THREADS, 0, s>>>(A, tm, tn);
  else k_matmul<S, kNone><<<grid, S::THREADS, 0, s>>>(A, tm, tn);
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

template <int TYPE>
hipError_t matmul_of(const MatmulArgs &A, hipStream_t s) {
  switch (best_tile(A.M, A.N, A.K)) {
    case 0: return matmul_as<TYPE, 16, 16, 16, 16, 512, 8, 4>(A, s);
    case 1: return matmul_as<TYPE, 16, 32, 16, 16, 512, 4, 3>(A, s);
    case 2: return matmul_as<TYPE, 32, 32, 16, 16, 512, 2, 4>(A, s);
    case 3: return matmul_as<TYPE, 64, 32, 32, 16, 512, 2, 3>(A, s);
    case 4: return matmul_as<TYPE, 64, 64, 32, 32, 256, 2, 4>(A, s);
    case 5: return matmul_as<TYPE, 128, 64, 32, 32, 128, 1, 3>(A, s);
    case 6: return matmul_as<TYPE, 128, 128, 32, 64, 128, 1, 3>(A, s);
    case 7: return matmul_as<TYPE, 256, 128, 64, 64, 128, 1, 3>(A, s);
    default: return matmul_as<TYPE, 256, 256, 128, 64, 128, 1, 2>(A, s);
  }
}

template <int TYPE, int BN, int WK, int NS>
hipError_t few_as(const QuantizeArgs &X, const MatmulArgs &A, int64_t rows_bytes, hipStream_t s) {
  using S = Shape<TYPE, 16, BN, 16, 16, 512, WK, NS>;
  constexpr int RING = S::NS * S::BN * S::BK;
  static_assert(RING >= S::WAVES * S::NT * 1024, "the parts' sums fit the ring");
  static_assert(S::THREADS == kFewThreads, "whole loads of a row");
  // more than 64 KB of LDS asked for at the launch
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_linear_few<S>), hipFuncAttributeMaxDynamicSharedMemorySize, kFewBytes);
  if (e != hipSuccess) return e;
  const int tiles = (A.N + BN - 1) / BN;
  k_linear_few<S><<<(tiles + 7) / 8 * 8, S::THREADS, (size_t)(RING + rows_bytes), s>>>(X, A, tiles);
  return hipGetLastError();
}

// Where one launch is faster than two: a block a CU or less, or a single row
// and two blocks a CU.  (bfloat16, eight sets of weights in turn, us of one
// launch and of two: 1 x 7168 x 5120 8.9 and 11.6, 4 rows 10.4 and 11.6; 1 x 896
// x 5120 5.3 and 7.3; 1 x 5120 x 640 4.1 and 7.3; 1 x 5120 x 20480 23.5 and 28.6;
// 1 x 10240 x 5120 12.9 and 16.2; 4 x 10240 x 5120 18.9 and 16.2, where every CU
// makes the codes twice.)
template <int TYPE>
bool few_of(const QuantizeArgs &X, const MatmulArgs &A, hipStream_t s, hipError_t *e) {
  const int64_t size = X.type == kF32 ? 4 : 2, load = kFewThreads * 16;
  const int64_t bytes = A.M * ((A.K * size + load - 1) / load * load + (A.K + 511) / 512 * 512 + 64);
  if (A.N <= 256 * 16 && 6 * 8192 + bytes <= kFewBytes) *e = few_as<TYPE, 16, 8, 6>(X, A, bytes, s);
  else if (A.N <= 256 * 32 && 4 * 16384 + bytes <= kFewBytes) *e = few_as<TYPE, 32, 4, 4>(X, A, bytes, s);
  else if (A.M == 1 && 3 * 16384 + bytes <= 80 << 10 && A.N <= kMostBlocks * 32) *e = few_as<TYPE, 32, 4, 3>(X, A, bytes, s);
  else return false;
  return true;
}

}  // namespace

bool launch_linear_few(const QuantizeArgs &X, const MatmulArgs &A, hipStream_t s, hipError_t *e) {
  const int64_t size = X.type == kF32 ? 4 : 2;
  if (A.M > kFewRows || A.K < 16 || A.K % 16 || A.w_stride > (1 << 23)) return false;
  // loads of 16 bytes, of a row's own
  if (((uintptr_t)X.x | (uintptr_t)(A.M > 1 ? X.x_stride * size : 0) | (uintptr_t)A.w | (uintptr_t)A.w_stride) & 15) return false;
  return A.out_type == kF32 ? few_of<kF32>(X, A, s, e) : A.out_type == kF16 ? few_of<kF16>(X, A, s, e) : few_of<kBF16>(X, A, s, e);
}

hipError_t launch_quantize_rows(const QuantizeArgs &A, hipStream_t s) {
  return A.type == kF32 ? quantize_of<kF32>(A, s) : A.type == kF16 ? quantize_of<kF16>(A, s) : quantize_of<kBF16>(A, s);
}

bool matmul_fits(int32_t M, int32_t N, int32_t K) {
  const Tile &t = kTiles[best_tile(M, N, K)];
  return ((int64_t)(M - 1) / t.bm + 1) * ((N - 1) / t.bn + 1) <= kMostBlocks;
}

hipError_t launch_scaled_matmul(const MatmulArgs &A, hipStream_t s) {
  return A.out_type == kF32 ? matmul_of<kF32>(A, s) : A.out_type == kF16 ? matmul_of<kF16>(A, s) : matmul_of<kBF16>(A, s);
}

}  // namespace fs
