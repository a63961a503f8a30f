// fs_attention.hip -- causal attention over the paged 8-bit cache.
//
// o_i = sum_j softmax_j(scale <q_i, K_j>) V_j with K_j = kscale * kcode_j and
// V_j = vscale * vcode_j.  One pass over the tokens with the running maximum
// and sum; the context is cut over blocks, and of the blocks that have parts
// of a row tile the last to arrive adds them up.
#include <algorithm>
#include <atomic>
#include <chrono>
#include <type_traits>

#include "fs_serving.h"

namespace fs {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kFloor = -3.40282347e38f;  // a maximum over no tokens: finite, so differences are no NaN, and above no logit
constexpr int kTile = 64;         // tokens of one step of a wavefront

// The larger of a lane's value and of the one 32 (or 16) lanes on.
__device__ __forceinline__ float max_over_32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_over_16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// ------------------------------------------------------------ who does what --
// An item is a tile of R rows of one sequence and cache head; a row is a (new
// token, query head of the group) pair.  An item has as many units of work as
// its sequence has 64-token tiles that some query sees (causal rows see fewer:
// early and late row tiles alternate, which evens that out).  The units of all
// items in a row are cut into equal runs, one a block, wherever the cuts fall,
// so that ragged lengths leave no block with more to do.  A block writes an
// item that lies within its run, and the unnormalised part of one that does
// not: at most two, one at either end.  The last block to write a part of an
// item adds them up, in their order, so that results do not depend on which
// block that is.
// All of this follows from the lengths alone, and each block derives it.
// (Units are counted in 32 bits: launch_cache_attention sees to their number.)

// Rows to (token, head of the group): a row tile's first row is divided once,
// the few from there on by a multiplication (exact while group + 256 rows
// times group stay below 2^32).
struct Rows {
  int token, head;  // of the first row
  uint32_t group, per;

  __device__ __forceinline__ Rows(int r0, int g, uint32_t inverse) : group(g), per(inverse) {
    token = r0 / g;
    head = r0 - token * g;
  }
  __device__ __forceinline__ int2 operator()(int i) const {
    const uint32_t x = head + i, t = group == 1 ? x : __umulhi(x, per);
    return {token + (int)t, (int)(x - t * group)};
  }
};

constexpr int kItemUnits = 8;

struct Seq {
  int q0, n;   // first row of q, new tokens
  int length;  // tokens in the cache
  int t0;      // first tile that some query sees
  int units;   // tiles from there on; at least kItemUnits, which an item costs in any case
};

__device__ __forceinline__ Seq sequence(const AttendArgs &A, int s) {
  Seq q;
  q.q0 = min(max(A.cu_q[s], 0), A.n_tokens);
  q.n = min(min(max(A.cu_q[s + 1], q.q0), A.n_tokens) - q.q0, A.max_q);
  const int64_t room = min(A.table_width << A.c.page_shift, (int64_t)0x7fffffc0);
  q.length = (int)min((int64_t)max(A.ctx_lens[s], 0), room);
  const int64_t first = (int64_t)q.length - q.n;
  const int64_t from = A.window ? max((int64_t)0, first - A.window + 1) : 0;
  q.t0 = (int)(from / kTile);
  q.units = max(kItemUnits, (int)(((int64_t)q.length + kTile - 1) / kTile) - q.t0);
  return q;
}

// What a kernel takes: sequences of lo .. hi - 1 rows, in runs of at least
// `least` units.  An item's units are rounded up to a multiple of round + 1 (a
// power of two): where that is the length of a run, no block has the end of an
// item and the start of the next.
struct Share {
  int least, lo, hi, round;
};

// Units of an item of a sequence.
__device__ __forceinline__ uint32_t item_units(const Seq &q, const Share &w) { return (uint32_t)(q.units + w.round) & ~(uint32_t)w.round; }

__device__ __forceinline__ int row_tiles(const Seq &q, int group, int R, const Share &w) {
  const int64_t rows = (int64_t)q.n * group;
  return rows < w.lo || rows >= w.hi ? 0 : (int)((rows + R - 1) / R);
}

// Prefix sums of the sequences' units (pre, in LDS) and their total; all
// threads of the block call it.  Where cu_q falls sequences overlap and may have
// more units than launch_cache_attention allows for: sums that pass 32 bits stay
// at their largest, and such a call does nothing.
template <int THREADS, int R>
__device__ uint32_t list_units(const AttendArgs &A, int group, const Share &share, uint32_t *pre) {
  __shared__ uint32_t carry[THREADS / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t base = 0;
  for (int s0 = 0; s0 < A.n_seqs; s0 += THREADS) {
    const int s = s0 + threadIdx.x;
    uint32_t v = 0;
    if (s < A.n_seqs) {
      const Seq q = sequence(A, s);
      v = (uint32_t)(A.c.n_heads * row_tiles(q, group, R, share)) * item_units(q, share);
    }
    uint32_t sum = v;
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t x = (uint32_t)__shfl_up((int)sum, o);
      if (lane >= o) sum = __builtin_elementwise_add_sat(sum, x);
    }
    if (lane == 63) carry[wave] = sum;
    __syncthreads();
    uint32_t before = base;
    for (int i = 0; i < THREADS / 64; ++i) {
      if (i < wave) before += carry[i];
      base = __builtin_elementwise_add_sat(base, carry[i]);
    }
    if (s < A.n_seqs) pre[s] = before + sum - v;
    __syncthreads();
  }
  return base > 0x7fffffffu ? 0 : base;
}

__device__ __forceinline__ uint32_t run_length(uint32_t total, uint32_t blocks, const Share &share) {
  return max((total + blocks - 1) / blocks, (uint32_t)share.least);
}

struct Item {
  int s, h, r0;       // sequence, cache head, first row
  uint32_t start;     // its first unit
  uint32_t units;
  Seq q;
};

// The item of a unit.  Sequences without units share their prefix with the
// next, so the last one whose prefix is at most `unit` has it.
template <int R>
__device__ __forceinline__ Item item_at(const AttendArgs &A, int group, const Share &share, const uint32_t *pre, uint32_t unit) {
  int lo = 0, hi = A.n_seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= unit) lo = mid;
    else hi = mid;
  }
  Item it;
  it.s = lo;
  it.q = sequence(A, lo);
  it.units = item_units(it.q, share);
  const uint32_t rel = unit - pre[lo], at = rel / it.units;
  it.start = pre[lo] + at * it.units;
  const uint32_t tiles = row_tiles(it.q, group, R, share), k = at % tiles;
  it.h = (int)(at / tiles);
  it.r0 = (int)(k & 1 ? tiles - 1 - k / 2 : k / 2) * R;
  return it;
}

// Blocks of the row kernel: two a CU of four wavefronts or one of eight; of the
// other: one a CU.
constexpr int kRowBlocks = 512, kChunkBlocks = 256;
constexpr int row_blocks(int waves) { return kRowBlocks * 4 / waves; }
static_assert(kRowBlocks < 4096, "counts of parts have 12 bits");

// A cut costs a block about as much as 16 tiles.  Items that are small beside
// a run, or where runs are short not much longer, are not cut: a cut within
// one moves to its nearer end.
__device__ __forceinline__ bool stays_whole(uint32_t units, uint32_t run) {
  return units * 4 <= run || (run < 24 && units <= 2 * run);
}

// The units of an item that a run up to `stop` does, from `unit` on (which
// moves past them); false if there are none.
__device__ __forceinline__ bool take(const Item &it, uint32_t run, uint32_t stop, uint32_t &unit, uint32_t &from, uint32_t &to) {
  const uint32_t end = it.start + it.units;
  from = unit - it.start;
  to = min(it.units, from + stop - unit);
  if (stays_whole(it.units, run)) {
    const bool of_last = from > 0 && 2 * from >= it.units;                      // the run before has it
    const bool of_next = stop < end && 2 * (stop - it.start) < it.units;        // the one after
    from = 0;
    to = it.units;
    unit = end;
    return !of_last && !of_next;
  }
  unit += to - from;
  return true;
}

// The first token that a query at position p sees: positions may be negative and
// windows up to 2^31 - 1, whose difference has no 32 bits.
__device__ __forceinline__ int first_seen_from(const AttendArgs &A, int p) {
  return A.window && p >= A.window ? p - A.window + 1 : 0;
}

// The tiles of units from .. to - 1 of an item whose rows belong to the
// sequence's new tokens j0 .. j1 that some of them see.
__device__ __forceinline__ int2 tiles_of(const AttendArgs &A, const Seq &q, int j0, int j1, bool whole, int from, int to) {
  const int first = q.length - q.n, end = min(q.length, first + j1 + 1);
  const int low = first_seen_from(A, first + j0);
  if (end <= low) return {0, 0};
  const int a = low / kTile, b = (end + kTile - 1) / kTile;
  if (whole) return {a, b};
  return {max(a, q.t0 + from), min(b, q.t0 + to)};
}

// Workspace: a counter a run, then of each part of an item the rows' maximum
// and sum and their unnormalised outputs.
constexpr int kRows = 16;
__host__ __device__ constexpr int64_t part_floats(int R, int D) { return (int64_t)R * (D + 2); }
// A run's part of the item that it starts in the middle of, or that it leaves.
__device__ __forceinline__ int64_t part_index(uint32_t run, bool from_start) { return 2 * (int64_t)run + from_start; }
struct Parts {
  unsigned long long *arrived;  // of the item that goes on beyond a run, by the run that it starts in
  float *floats;
  // The workspace comes with any contents, so a count is one only under the
  // call's own number (52 bits, above 12 of the count); the last to arrive
  // leaves 0, for a graph that runs the call again.
  unsigned long long call;  // 0: the parts are left to k_join
};

// Workgroups go round the eight XCDs in turn: each XCD gets neighbouring runs
// (grids are multiples of eight), so that row tiles of one head meet in its L2,
// and the same number of them, however few there are (us a call, with the first
// XCDs full and so: 24 users of 1000 tokens on 8 heads 15.8 and 14.1, 140 of up to
// 1000 on two 16.9 and 15.3, 32 of up to 8000 on one 17.9 and 16.9).  A block
// beyond the runs gets one that starts past the units.
template <uint32_t BLOCKS>
__device__ __forceinline__ uint32_t run_of_block(uint32_t total, uint32_t run) {
  // at least total / run / 8, which is at most BLOCKS / 8 (the factor is for the rounding)
  const float share = (float)total * __builtin_amdgcn_rcpf((float)run) * (0.125f * 1.00001f);
  const uint32_t per = min(BLOCKS / 8, (uint32_t)share + 1), at = blockIdx.x >> 3;
  return at < per ? (blockIdx.x & 7) * per + at : BLOCKS;
}

// Parts go from block to block, whose L2 may be another XCD's: they are stored
// and read at the device's scope, two floats at a time, past the L2.  (A fence
// would write back or drop all of an L2: 64 users 281 us instead of 80.)
__device__ __forceinline__ void put(float *to, float a, float b) {
  const unsigned long long v = __float_as_uint(a) | (unsigned long long)__float_as_uint(b) << 32;
  __hip_atomic_store((unsigned long long *)to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get(const float *from) {
  const unsigned long long v =
      __hip_atomic_load((unsigned long long *)from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return {__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
}

// Whether this block is the last of `parts` to have written its part.
__device__ __forceinline__ bool last_to_arrive(const Parts &P, uint32_t b0, int parts) {
  __shared__ int last;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // each wavefront's stores are done before the block counts as there
  __syncthreads();
  if (threadIdx.x == 0) {
    unsigned long long *const slot = P.arrived + b0;
    unsigned long long seen = __hip_atomic_load(slot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), now;
    for (;;) {
      now = ((seen & ~0xfffull) == P.call ? seen : P.call) + 1;
      const unsigned long long was = atomicCAS(slot, seen, now);
      if (was == seen) break;
      seen = was;
    }
    last = (int)(now & 0xfff) == parts;
    if (last) atomicExch(slot, 0ull);
  }
  __syncthreads();
  return last;
}

// Four neighbouring elements of row i from d on, to where they go.
template <int TYPE, int D>
__device__ __forceinline__ void store_joined(const AttendArgs &A, const Item &it, const Rows &of, int i, int d, float4v out, float sum) {
  const int2 to = of(i);
  uint16_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = bits16<TYPE>(sum == 0.0f ? 0.0f : out[j] / sum);
  __builtin_memcpy((uint16_t *)A.out + ((int64_t)(it.q.q0 + to.x) * A.n_q_heads + it.h * (int)of.group + to.y) * D + d, w, 8);
}

// Adds up the parts of an item of many rows: four times four elements a lane and
// two parts at a time, so that loads enough are under way.  (2048 tokens of 40
// heads over 8192: 426 us, 438 with the loop for few rows below; two such 667 and
// 682; 512 of 40 heads over 4096 beside 32 users 134 and 145.)
template <int TYPE, int D, int R, int WAVES>
__device__ void join_many(const AttendArgs &A, const Item &it, const Rows &of, int rows, uint32_t b0, int parts, const float *floats) {
  constexpr int HELD = 4, STEP = 64 * WAVES;
  const int pieces = rows * (D / 4);
  for (int at = threadIdx.x; at < pieces; at += HELD * STEP) {
    float M[HELD], sum[HELD];
    float4v out[HELD];
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
      M[h] = kFloor;
      sum[h] = 0.0f;
      out[h] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    }
    for (int p0 = 0; p0 < parts; p0 += 2) {
      float2 ml[2][HELD], v0[2][HELD], v1[2][HELD];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int p = min(p0 + j, parts - 1);
        const float *const f = floats + part_index(b0 + p, p == 0) * part_floats(R, D);
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
          const int e = min(at + h * STEP, pieces - 1), i = e / (D / 4), d = e % (D / 4) * 4;
          ml[j][h] = get(f + 2 * i);
          v0[j][h] = get(f + 2 * R + i * D + d);
          v1[j][h] = get(f + 2 * R + i * D + d + 2);
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (p0 + j >= parts) break;
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
          const float m_new = fmaxf(M[h], ml[j][h].x);
          const float keep = __builtin_amdgcn_exp2f(M[h] - m_new), add = __builtin_amdgcn_exp2f(ml[j][h].x - m_new);
          sum[h] = sum[h] * keep + ml[j][h].y * add;
          out[h] = out[h] * keep + float4v{v0[j][h].x, v0[j][h].y, v1[j][h].x, v1[j][h].y} * add;
          M[h] = m_new;
        }
      }
    }
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
      const int e = at + h * STEP;
      if (e < pieces) store_joined<TYPE, D>(A, it, of, e / (D / 4), e % (D / 4) * 4, out[h], sum[h]);
    }
  }
  __syncthreads();
}

// The same for an item of few rows, four elements a lane.  Where there are many
// parts the wavefronts share them.
template <int TYPE, int D, int R, int WAVES>
__device__ void join(const AttendArgs &A, const Item &it, const Rows &of, int rows, uint32_t b0, int parts, const float *floats) {
  __shared__ float lm[WAVES][64], ll[WAVES][64];
  __shared__ float4v lo[WAVES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool together = parts > 8;
  const int pieces = rows * (D / 4), step = together ? 64 : 64 * WAVES;
  for (int at = together ? 0 : wave * 64; at < pieces; at += step) {
    const int e = min(at + lane, pieces - 1), i = e / (D / 4), d = e % (D / 4) * 4;
    float M = kFloor, sum = 0.0f;
    float4v out = {0.0f, 0.0f, 0.0f, 0.0f};
    // many loads under way at a time; beyond the last part, the last again with no weight
    constexpr int AHEAD = 8;
    const int p_step = together ? WAVES : 1;
    for (int p0 = together ? wave : 0; p0 < parts; p0 += AHEAD * p_step) {
      float2 ml[AHEAD], v0[AHEAD], v1[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int p = min(p0 + j * p_step, parts - 1);
        const float *const f = floats + part_index(b0 + p, p == 0) * part_floats(R, D);
        ml[j] = get(f + 2 * i);
        v0[j] = get(f + 2 * R + i * D + d);
        v1[j] = get(f + 2 * R + i * D + d + 2);
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        if (p0 + j * p_step >= parts) break;
        const float m_new = fmaxf(M, ml[j].x);
        const float keep = __builtin_amdgcn_exp2f(M - m_new), add = __builtin_amdgcn_exp2f(ml[j].x - m_new);
        sum = sum * keep + ml[j].y * add;
        out = out * keep + float4v{v0[j].x, v0[j].y, v1[j].x, v1[j].y} * add;
        M = m_new;
      }
    }
    if (together) {
      lm[wave][lane] = M;
      ll[wave][lane] = sum;
      lo[wave][lane] = out;
      __syncthreads();
      for (int w = 0; w < WAVES; ++w) M = fmaxf(M, lm[w][lane]);
      sum = 0.0f;
      out = float4v{0.0f, 0.0f, 0.0f, 0.0f};
      for (int w = 0; w < WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f(lm[w][lane] - M);
        sum += f * ll[w][lane];
        out += f * lo[w][lane];
      }
      __syncthreads();
    }
    if (at + lane < pieces && (!together || wave == 0)) {
      store_joined<TYPE, D>(A, it, of, i, d, out, sum);
    }
  }
  __syncthreads();
}

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

// Four sums with 128 in them to their second bytes, and their first as signed.
__device__ __forceinline__ int2 split_bytes(const uint32_t (&b)[4]) {
  const uint32_t u = __builtin_amdgcn_perm(b[1], b[0], 0x05010400), v = __builtin_amdgcn_perm(b[3], b[2], 0x05010400);
  return {(int)__builtin_amdgcn_perm(v, u, 0x07060302), (int)(__builtin_amdgcn_perm(v, u, 0x05040100) ^ 0x80808080u)};
}

// ONE: pages of 64 tokens, so a tile is a page and its address is scalar.
template <int TYPE, int D, int WAVES, bool ONE>
__global__ __launch_bounds__(64 * WAVES, 2) void k_attend_rows(AttendArgs A, Share share, Parts P) {
  constexpr int STEPS = D / 64, DT = D / 16;
  extern __shared__ uint32_t pre[];
  __shared__ float lo[WAVES][kRows][D + 4];
  __shared__ float lm[WAVES][kRows], ll[WAVES][kRows];
  const Cache &c = A.c;
  const int group = A.n_q_heads / c.n_heads;
  const uint32_t total = list_units<64 * WAVES, kRows>(A, group, share, pre), run = run_length(total, gridDim.x, share);
  const uint32_t mine = run_of_block<row_blocks(WAVES)>(total, run);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = lane & 15, G = lane >> 4, kg = row >> 2;
  const int PS = ONE ? 64 : 1 << c.page_shift;

  const uint32_t stop = min((mine + 1) * run, total);
  for (uint32_t unit = mine * run; unit < stop;) {
    const Item it = item_at<kRows>(A, group, share, pre, unit);
    const Seq &q = it.q;
    const int s = it.s, h = it.h, r0 = it.r0, rows = min(kRows, q.n * group - r0);
    uint32_t from, to;
    if (!take(it, run, stop, unit, from, to)) continue;
    const bool whole = from == 0 && to == it.units;
    const Rows of(r0, group, A.per_group);
    const int2 mine_of = of(row);  // (token, head of the group)
    const int j1 = of(rows - 1).x;
    const int2 span = tiles_of(A, q, of.token, j1, whole, (int)from, (int)to);
    const int first = q.length - q.n;
    const int token = row < rows ? mine_of.x : 0, q_head = h * group + mine_of.y;
    // what this row sees, what some row sees, what all do
    const int last_seen = row < rows ? first + token : -1;
    const int first_seen = first_seen_from(A, last_seen);
    const int all_top = first + of.token, top = first + j1;
    const int low = first_seen_from(A, all_top), all_low = first_seen_from(A, top);
    const int page_top = max(top, 0) >> c.page_shift, page_low = min(low, max(top, 0)) >> c.page_shift;
    const int32_t *const table = A.table + s * A.table_width;

    int32_t id_k = 0, id_v = 0;  // table entries as loaded: what is made of them waits for them
    const auto pages = [&](int tile) {
      if constexpr (ONE) {
        id_k = id_v = table[min(max(tile, page_low), page_top)];
      } else {
        const int tok = tile * kTile;
        id_k = table[min(max((tok + kg * 16) >> c.page_shift, page_low), page_top)];
        id_v = table[min(max((tok + G * 16) >> c.page_shift, page_low), page_top)];
      }
    };
    // One place for a tile's keys and one for its values: the next tile's are
    // asked for as soon as this one's have been multiplied.  (With two places for
    // whole tiles, and the loop's body twice, 4 users of 131072 tokens took 53.7
    // us instead of 50.0, 64 of 512 to 8192 74.6 instead of 73.5.)
    const auto page = [&](int32_t id) { return (int64_t)min((uint32_t)id, (uint32_t)(c.n_pages - 1)) * c.n_heads + h; };
    int4v tk[4][STEPS], tv[DT];
    float next_ks = 0.0f, next_vs = 0.0f;
    const auto fetch_k = [&](int tile) {
      const int64_t pk = page(id_k), pv = page(id_v);
      const int at_k = ONE ? kg * 16 : (tile * kTile + kg * 16) & (PS - 1);
      const int8_t *const kp = c.k + pk * (PS * D) + ((at_k + (row & 3)) * D + G * 16);
      next_ks = c.k_scale[pv];
      next_vs = c.v_scale[pv];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int st = 0; st < STEPS; ++st) tk[i][st] = *(const int4v *)(kp + i * 4 * D + st * 64);
    };
    const auto fetch_v = [&](int tile) {
      const int at_v = ONE ? G * 16 : (tile * kTile + G * 16) & (PS - 1);
      const int8_t *const vp = c.v + page(id_v) * (PS * D) + (row * PS + at_v);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) tv[dt] = *(const int4v *)(vp + dt * 16 * PS);
    };
    int tile = span.x + wave;
    if (tile < span.y) {
      pages(tile);
      fetch_k(tile);
      fetch_v(tile);
      if (tile + WAVES < span.y) pages(tile + WAVES);
    }

    // the row's codes, 15 bits against its largest: in the low bits of a sum
    // with 1.5 * 2^23 + 128 (the 128 makes the low byte signed)
    int4v q_hi[STEPS], q_lo[STEPS];
    float q_step;
    {
      using ushort2v = unsigned short __attribute__((ext_vector_type(2)));
      int4v raw[STEPS][2];
      ushort2v most = {0, 0};  // both types' magnitudes are in the order of their bits, a NaN's above all
#pragma unroll
      for (int st = 0; st < STEPS; ++st)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          raw[st][j] = int4v{0, 0, 0, 0};
          if (row < rows)
            raw[st][j] = load16((const uint16_t *)A.q + (int64_t)(q.q0 + token) * A.q_stride + q_head * D + st * 64 + G * 16 + j * 8);
        }
#pragma unroll
      for (int st = 0; st < STEPS; ++st)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            most = __builtin_elementwise_max(most, __builtin_bit_cast(ushort2v, raw[st][j][i] & 0x7fff7fff));
      int bits = max((int)most[0], (int)most[1]);
      bits = max(bits, __shfl_xor(bits, 16));
      bits = max(bits, __shfl_xor(bits, 32));
      const float largest = value16<TYPE>((uint16_t)bits);
      const float inverse = largest < kTiny ? 0.0f : 32512.0f / largest;
      // no code stands for an infinity, whose logits may cancel: as with a NaN all are NaN
      q_step = (largest < kTiny ? 0.0f : largest / 32512.0f + (largest - largest)) * (A.scale * kLog2e);
#pragma unroll
      for (int st = 0; st < STEPS; ++st)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t b[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint16_t word = (uint16_t)(raw[st][w >> 1][(w & 1) * 2 + (i >> 1)] >> 16 * (i & 1));
            b[i] = __float_as_uint(__builtin_fmaf(value16<TYPE>(word), inverse, 12582912.0f + 128.0f));
          }
          const int2 bytes = split_bytes(b);
          q_hi[st][w] = bytes.x;
          q_lo[st][w] = bytes.y;
        }
    }

    float4v o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    float m = kFloor, l = 0.0f;
    for (; tile < span.y; tile += WAVES) {
      const int base = tile * kTile;
      float sc[16];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        int4v hi = {0, 0, 0, 0}, low_sum = {0, 0, 0, 0};
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(tk[j][st], q_hi[st], hi, 0, 0, 0);
          low_sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(tk[j][st], q_lo[st], low_sum, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[j * 4 + i] = (float)(hi[i] * 256 + low_sum[i]);
      }
      // sc[i]: token base + G * 16 + i
      float ks = next_ks, vs = next_vs;
      const bool more = tile + WAVES < span.y;
      if (more) fetch_k(tile + WAVES);
      const bool edge = base < all_low || base + kTile - 1 > all_top;  // some row does not see all of it
      int least = first_seen - base - G * 16, most = last_seen - base - G * 16;
      if (edge && (most < 0 || least > 15)) {  // no page of this row's
        ks = 1.0f;
        vs = 0.0f;
      }
      const bool zero = vs < kZeroScale;
      const float lift = zero ? -60.0f : __builtin_amdgcn_logf(vs);
      const float per = zero ? 0x1p60f : 1.0f / vs;
      const float cq = __builtin_fmaf(q_step, ks, ks - ks);  // NaN under an infinite scale, whatever the sum's sign
      // Logits may reach 2^29 cq.  From 2^20 on a value scale would be lost in them:
      // it is added to their differences from the largest.
      const bool wild = __any(fabsf(cq) > 0x1p-9f);
      const float with = wild ? 0.0f : lift;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = __builtin_fmaf(sc[i], cq, with);
      if (edge) {
        asm volatile("" : "+v"(least), "+v"(most));  // keeps the comparisons in here
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = i >= least && i <= most ? sc[i] : -INFINITY;
      }
      float top_s = kFloor;
#pragma unroll
      for (int i = 0; i < 16; ++i) top_s = fmaxf(top_s, sc[i]);
      top_s = max_over_32(max_over_16(top_s));
      const float m_new = fmaxf(m, top_s);
      float below = top_s - m_new;
      if (wild) {
        const float most_lift = max_over_32(max_over_16(lift));
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = (sc[i] - top_s) + (lift - most_lift);
        top_s = 0.0f;
        below += most_lift;
      }
      const float keep = __builtin_amdgcn_exp2f(m - m_new), add = __builtin_amdgcn_exp2f(below);
      m = m_new;
      // probabilities against the tile's largest: 15-bit codes, in the low
      // bits of a sum with 2^23 + 128 (the 128 makes the low byte signed)
      const float full = zero ? 0.0f : 32512.0f;
      float sum = 0.0f;
      int4v p_hi, p_lo;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = __builtin_amdgcn_exp2f(sc[j * 4 + i] - top_s);
          sum += p;
          b[i] = __float_as_uint(__builtin_fmaf(p, full, 8388608.0f + 128.0f));
        }
        const int2 bytes = split_bytes(b);
        p_hi[j] = bytes.x;
        p_lo[j] = bytes.y;
      }
      l = l * keep + sum * per * add;
      if (__any(keep != 1.0f)) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] *= keep;
      }
      const float step = add * (1.0f / 32512.0f);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const int4v none = {0, 0, 0, 0};
        const int4v hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(tv[dt], p_hi, none, 0, 0, 0);
        const int4v low_sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(tv[dt], p_lo, none, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          o[dt][i] = __builtin_fmaf((float)(hi[i] * 256 + low_sum[i]), step, o[dt][i]);
      }
      if (more) {
        fetch_v(tile + WAVES);
        if (tile + 2 * WAVES < span.y) pages(tile + 2 * WAVES);
      }
    }
    // the row's sum over the four lanes that hold it, then the wavefronts
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (G == 0) {
      lm[wave][row] = m;
      ll[wave][row] = l;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *(float4v *)&lo[wave][row][dt * 16 + G * 4] = o[dt];
    __syncthreads();
    for (int e = threadIdx.x; e < rows * (D / 2); e += 64 * WAVES) {
      const int i = e / (D / 2), d = e % (D / 2) * 2;
      float M = lm[0][i];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) M = fmaxf(M, lm[w][i]);
      float sum = 0.0f, out0 = 0.0f, out1 = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f(lm[w][i] - M);
        sum += f * ll[w][i];
        out0 += f * lo[w][i][d];
        out1 += f * lo[w][i][d + 1];
      }
      if (!whole) {
        float *const part = P.floats + part_index(mine, from == 0) * part_floats(kRows, D);
        if (d == 0) put(part + 2 * i, M, sum);
        put(part + 2 * kRows + i * D + d, out0, out1);
      } else {
        const int2 at = of(i);
        const uint16_t w[2] = {bits16<TYPE>(sum == 0.0f ? 0.0f : out0 / sum), bits16<TYPE>(sum == 0.0f ? 0.0f : out1 / sum)};
        __builtin_memcpy((uint16_t *)A.out + ((int64_t)(q.q0 + at.x) * A.n_q_heads + h * group + at.y) * D + d, w, 4);
      }
    }
    if (whole || P.call == 0) {
      __syncthreads();
    } else {
      const uint32_t b0 = it.start / run, b1 = (it.start + it.units - 1) / run;  // the runs that have parts of it
      if (last_to_arrive(P, b0, (int)(b1 - b0 + 1)))
        join<TYPE, D, kRows, WAVES>(A, it, of, rows, b0, (int)(b1 - b0 + 1), P.floats);
    }
  }
}

// ------------------------------------------------- many rows, binary16 products --
// A block takes 256 rows, 32 a wavefront, and 64 tokens at a time, whose codes
// it turns into binary16 in LDS once for all rows (exactly: codes are small
// integers), two tiles ahead.  A step has two parts, the products (of the
// tile's keys, and of the values of the tile before) and the exponentials; one
// of the two wavefronts of a SIMD is a part behind the other, so that one
// multiplies while the other takes exponentials.  S^T = K Q^T and
// O^T = V^T P^T with 32 x 32 x 16 products: a lane has one row, and K's rows
// are dealt so that its eight tokens of each 16 are neighbours, which makes
// the probabilities the second operand of the second product as they stand.
//
// Queries are scaled by a power of two, below 2 in magnitude, before they are
// rounded to binary16 (bfloat16 ones exactly, but for elements under 2^-14 of
// the row's largest).  The maximum that probabilities are taken against may
// lag by 2^8, so the output is seldom rescaled; with 2^6 on top probabilities
// reach 2^14 and keep 11 bits down to 2^-20 of the largest.
constexpr int kChunkRows = 256, kChunkThreads = 512, kChunkLeast = 128;
constexpr float kLag = 8.0f, kLift = 6.0f;

// The block's barrier after this wavefront's LDS accesses; its loads go on.
__device__ __forceinline__ void part_end() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// N products with an operand each from LDS, read AHEAD products ahead, which
// covers the reads' latency (left to itself the compiler reads, waits and
// multiplies in turn).
// `between` is done while products are under way.
template <int N, int AHEAD, class Read, class Multiply, class Between>
__device__ __forceinline__ void products(Read read, Multiply multiply, Between between) {
  half8 held[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) held[i] = read(i);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    multiply(i, held[i % AHEAD]);
    if (i + AHEAD < N) held[i % AHEAD] = read(i + AHEAD);
    between(i);
  }
}

// Four codes to binary16, two words: 1024 + (code + 128) is the byte under 0x64.
__device__ __forceinline__ int2 widen(int codes) {
  using half2v = _Float16 __attribute__((ext_vector_type(2)));
  const half2v bias = {(_Float16)-1152.0f, (_Float16)-1152.0f};
  const uint32_t b = (uint32_t)codes ^ 0x80808080u;
  const half2v x = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400)) + bias;
  const half2v y = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402)) + bias;
  return {__builtin_bit_cast(int, x), __builtin_bit_cast(int, y)};
}

// ONE: pages of 64 tokens, so a tile is a page and its address is scalar.
template <int TYPE, int D, bool ONE>
__global__ __launch_bounds__(kChunkThreads, 2) void k_attend_chunk(AttendArgs A, Share share, Parts P) {
  constexpr int kAhead = 6;
  constexpr int KK = D / 16, DT = D / 32, KC = D / 8;  // KC: 16-byte chunks of a token's binary16 keys
  extern __shared__ uint32_t pre[];
  __shared__ int4v lk[4][kTile * KC], lv[4][D * 8];
  __shared__ float4v scales[4][4];  // of 16 tokens: key scale, log2 and inverse of the value scale
  const Cache &c = A.c;
  const int group = A.n_q_heads / c.n_heads;
  const uint32_t total = list_units<kChunkThreads, kChunkRows>(A, group, share, pre), run = run_length(total, gridDim.x, share);
  const uint32_t mine = run_of_block<kChunkBlocks>(total, run), stop = min((mine + 1) * run, total);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int PS = ONE ? 64 : 1 << c.page_shift;
  // this thread's piece of a tile: 16 elements of a token's keys, 16 tokens of an element's values
  const int piece = D == 128 ? threadIdx.x : threadIdx.x & 255;
  const bool of_k = D == 128 || threadIdx.x < 256, of_v = D == 128 || threadIdx.x >= 256;
  const int k_token = piece / KK, k_part = piece % KK, v_row = piece >> 2, v_group = piece & 3;
  const auto k_place = [](int token, int chunk) {
    return token * KC + (chunk ^ (D == 128 ? token & 15 : (token >> 1) & 7));
  };
  const auto v_place = [](int d, int chunk) { return d * 8 + (chunk ^ ((d >> 1) & 7)); };

  for (uint32_t unit = mine * run; unit < stop;) {
    const Item it = item_at<kChunkRows>(A, group, share, pre, unit);
    const Seq &q = it.q;
    const int s = it.s, h = it.h, r0 = it.r0, rows = min(kChunkRows, q.n * group - r0);
    uint32_t from, to;
    if (!take(it, run, stop, unit, from, to)) continue;
    const bool whole = from == 0 && to == it.units;
    const Rows of(r0, group, A.per_group);
    const int2 mine_of = of(wave * 32 + col);  // (token, head of the group)
    const int j1 = of(rows - 1).x;
    const int2 span = tiles_of(A, q, of.token, j1, whole, (int)from, (int)to);
    const int first = q.length - q.n;
    const bool live = wave * 32 + col < rows;
    const int token = live ? mine_of.x : 0, q_head = h * group + (live ? mine_of.y : 0);
    const int last_seen = live ? first + token : -1;
    const int first_seen = first_seen_from(A, last_seen);
    // tiles that some row of this wavefront sees
    const int wave_rows = min(32, rows - wave * 32);
    const int wave_first = of(wave * 32).x, wave_last = of(wave * 32 + max(wave_rows, 1) - 1).x;
    const int wave_top = wave_rows > 0 ? first + wave_last : -1;
    const int wave_low = wave_rows > 0 ? first_seen_from(A, first + wave_first) : 0;
    // tokens that all of its rows see
    const int all_top = wave_rows > 0 ? first + wave_first : -1;
    const int all_low = first_seen_from(A, wave_top);
    // pages that some row of the block sees
    const int top = first + j1;
    const int low = first_seen_from(A, first + of.token);
    const int page_top = max(top, 0) >> c.page_shift, page_low = min(low, max(top, 0)) >> c.page_shift;
    const int32_t *const table = A.table + s * A.table_width;
    const auto entry = [&](int tok) { return table[min(max(tok >> c.page_shift, page_low), page_top)]; };
    const auto page_of = [&](int32_t id) { return (int64_t)min((uint32_t)id, (uint32_t)(c.n_pages - 1)) * c.n_heads + h; };

    // the row in binary16
    half8 qf[KK];
    float q_step;
    {
      int4v raw[KK];
      uint32_t most = 0;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        raw[kk] = int4v{0, 0, 0, 0};
        if (live) raw[kk] = load16((const uint16_t *)A.q + (int64_t)(q.q0 + token) * A.q_stride + q_head * D + kk * 16 + half * 8);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          most = max(most, __float_as_uint(value16<TYPE>((uint16_t)(raw[kk][i >> 1] >> 16 * (i & 1)))) & 0x7fffffffu);
      }
      most = max(most, (uint32_t)__shfl_xor((int)most, 32));
      // by a power of two near the largest; rows below 2^-100 count as zero
      const uint32_t e = min(max(most >> 23, 27u), 253u);
      const float up = __uint_as_float((254 - e) << 23 | (A.scale < 0.0f ? 0x80000000u : 0u)), down = __uint_as_float(e << 23);
      q_step = most >= 0x7f800000u ? NAN : down * (fabsf(A.scale) * kLog2e);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          qf[kk][i] = (_Float16)(value16<TYPE>((uint16_t)(raw[kk][i >> 1] >> 16 * (i & 1))) * up);
    }

    float16v o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = 0.0f;
    float m = kFloor, l = 0.0f;

    int32_t id_k = 0, id_v = 0;  // table entries, as loaded: what is made of them waits for them
    int4v codes_k, codes_v;
    float scale_k = 0.0f, scale_v = 0.0f;
    const auto pages = [&](int tile) {
      if constexpr (ONE) {
        id_k = id_v = table[min(max(tile, page_low), page_top)];
      } else {
        id_k = entry(tile * kTile + k_token);
        id_v = entry(tile * kTile + v_group * 16);
      }
    };
    const int k_at = ((k_token & (PS - 1)) * D) + k_part * 16, v_at = v_row * PS + (v_group * 16 & (PS - 1));
    const auto fetch = [&]() {
      const int64_t page_k = page_of(id_k), page_v = page_of(id_v);
      if (of_k) codes_k = *(const int4v *)(c.k + page_k * (PS * D) + k_at);
      if (of_v) codes_v = *(const int4v *)(c.v + page_v * (PS * D) + v_at);
      scale_v = c.v_scale[page_v];
      scale_k = c.k_scale[page_v];  // of threads 0 .. 3 the four groups'
    };
    // the codes fetched to binary16 in LDS, in eight steps
    int4v wide_k[2], wide_v[2];
    const auto deposit = [&](int buf, int step) {
      const int j = step & 3;
      if (step < 4 ? of_k : of_v) {
        const int2 w = widen(step < 4 ? codes_k[j] : codes_v[j]);
        int4v &to = (step < 4 ? wide_k : wide_v)[j >> 1];
        to[(j & 1) * 2] = w.x;
        to[(j & 1) * 2 + 1] = w.y;
        if (step == 3) {
          lk[buf][k_place(k_token, k_part * 2)] = wide_k[0];
          lk[buf][k_place(k_token, k_part * 2 + 1)] = wide_k[1];
        }
        if (step == 7) {
          if (scale_v < kZeroScale) wide_v[0] = wide_v[1] = int4v{0, 0, 0, 0};
          lv[buf][v_place(v_row, v_group * 2)] = wide_v[0];
          lv[buf][v_place(v_row, v_group * 2 + 1)] = wide_v[1];
        }
      }
      if (step == 7 && threadIdx.x < 4) {
        const bool none = scale_v < kZeroScale;
        // a NaN for an infinite key scale, whatever the sums' signs
        scales[buf][threadIdx.x] = float4v{scale_k + (scale_k - scale_k), none ? -60.0f : __builtin_amdgcn_logf(scale_v),
                                           none ? 0x1p60f : __builtin_amdgcn_rcpf(scale_v), 0.0f};
      }
    };
    const auto deposit_all = [&](int buf) {
#pragma unroll
      for (int step = 0; step < 8; ++step) deposit(buf, step);
    };
    const int last_tile = span.y - 1;
    if (span.x < span.y) {
      pages(span.x);
      fetch();
      pages(min(span.x + 1, last_tile));
      deposit_all(span.x & 3);
      fetch();
      pages(min(span.x + 2, last_tile));
      deposit_all((span.x + 1) & 3);
      fetch();
      pages(min(span.x + 3, last_tile));
    }
    half8 pf[4];
    bool waiting = false;  // pf holds the tile before
    const auto weigh = [&](int buf, auto between) {
      products<4 * DT, kAhead>(
          [&](int i) { return __builtin_bit_cast(half8, lv[buf][v_place(i % DT * 32 + col, i / DT * 2 + half)]); },
          [&](int i, half8 v) { o[i % DT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pf[i / DT], o[i % DT], 0, 0, 0); }, between);
    };
    part_end();
    if (wave >= 4) part_end();
    for (int tile = span.x; tile < span.y; ++tile) {
      const int base = tile * kTile, buf = tile & 3;
      const bool seen = base <= wave_top && base + kTile > wave_low;
      float16v sc[2];
      if (seen) {
        const int tok = (col >> 4) * 16 + ((col >> 2) & 1) * 8 + ((col >> 3) & 1) * 4 + (col & 3);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[t][i] = 0.0f;
        products<2 * KK, kAhead>(
            [&](int i) { return __builtin_bit_cast(half8, lk[buf][k_place(i % 2 * 32 + tok, i / 2 * 2 + half)]); },
            [&](int i, half8 k) { sc[i % 2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, qf[i / 2], sc[i % 2], 0, 0, 0); }, [](int) {});
      }
      // between the products tile + 2 goes to LDS: its place was last read a
      // step ago, and it is read two steps from here
      const int into = (tile + 2) & 3;
      if (waiting) {
        weigh((tile - 1) & 3, [&](int i) {
          if (i < 8) deposit(into, i);
        });
      } else {
        deposit_all(into);
      }
      waiting = seen;
      part_end();
      // the codes of tile + 3 (beyond the last the last again: with no
      // condition nothing waits for the loads here)
      fetch();
      pages(min(tile + 4, last_tile));
      if (seen) {
        // register i of tile t: token half * 8 + i % 8 of group g = 2 t + i / 8;
        // its logit (base 2, with the value scale) is x * slope[g] + add[g]
        float slope[4], add[4], per[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4v by = scales[buf][g];
          slope[g] = q_step * by[0];
          add[g] = by[1];
          per[g] = by[2];
        }
        if (base < all_low || base + kTile - 1 > all_top) {  // some row does not see all of it
          int least = first_seen - base - half * 8, most = last_seen - base - half * 8;
          asm volatile("" : "+v"(least), "+v"(most));  // keeps the comparisons in here
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            if (g * 16 - half * 8 > most || g * 16 + 15 - half * 8 < least) add[g] = per[g] = 0.0f;  // no page of this row's
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int at_i = (g & 1) * 8 + i, place = g * 16 + i;
              const float v = sc[g >> 1][at_i] * slope[g];
              sc[g >> 1][at_i] = place >= least && place <= most ? v : -INFINITY;
            }
            slope[g] = 1.0f;
          }
        }
        float top_s = kFloor;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int f = (g & 1) * 8;
          float most = fmaxf(sc[g >> 1][f], sc[g >> 1][f + 1]);
#pragma unroll
          for (int i = 2; i < 8; ++i) most = fmaxf(most, sc[g >> 1][f + i]);
          top_s = fmaxf(top_s, __builtin_fmaf(most, slope[g], add[g]));
        }
        top_s = max_over_32(top_s);
        // Logits so large that a rounding less would tell and a value scale would be
        // lost in them: as they are, the scale added to their differences from the largest.
        // (Past 2^27 the maximum holds none of the scale, and probabilities, with 2^14 over
        // one, hold value scales up to 2.)
        const bool wild = __any(fabsf(top_s) > 0x1p20f && top_s > kFloor);
        if (wild) {
          top_s = kFloor;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int at_i = (g & 1) * 8 + i;
              sc[g >> 1][at_i] *= slope[g];
              top_s = fmaxf(top_s, sc[g >> 1][at_i] + add[g]);
            }
            slope[g] = 1.0f;
          }
          top_s = max_over_32(top_s);
        }
        if (__any(top_s > m + kLag)) {
          const float m_new = fmaxf(m, top_s), keep = __builtin_amdgcn_exp2f(m - m_new);
          m = m_new;
          l *= keep;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] *= keep;
        }
        float less = m - kLift;
        if (wild) {
#pragma unroll
          for (int g = 0; g < 4; ++g) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int at_i = (g & 1) * 8 + i;
              sc[g >> 1][at_i] = (sc[g >> 1][at_i] - m) + add[g];
            }
            add[g] = kLift;
          }
          less = 0.0f;
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float plus = add[g] - less;
          float sum = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[g >> 1][(g & 1) * 8 + i], slope[g], plus));
            sum += p;
            pf[g][i] = (_Float16)p;
          }
          l = __builtin_fmaf(sum, per[g], l);
        }
      }
      part_end();
    }
    if (waiting) weigh(last_tile & 3, [](int) {});
    if (wave < 4) part_end();
    part_end();
    l += __shfl_xor(l, 32);
    if (live) {
      if (!whole) {
        float *const part = P.floats + part_index(mine, from == 0) * part_floats(kChunkRows, D);
        const int i = wave * 32 + col;
        if (half == 0) put(part + 2 * i, m, l);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float *const to = part + 2 * kChunkRows + (int64_t)i * D + dt * 32 + j * 8 + half * 4;
            put(to, o[dt][j * 4], o[dt][j * 4 + 1]);
            put(to + 2, o[dt][j * 4 + 2], o[dt][j * 4 + 3]);
          }
      } else {
        const float inverse = l == 0.0f ? 0.0f : 1.0f / l;
        uint16_t *const to = (uint16_t *)A.out + ((int64_t)(q.q0 + token) * A.n_q_heads + q_head) * D;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint16_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = bits16<TYPE>(o[dt][j * 4 + i] * inverse);
            __builtin_memcpy(to + dt * 32 + j * 8 + half * 4, w, 8);
          }
      }
    }
    if (!whole) {
      const uint32_t b0 = it.start / run, b1 = (it.start + it.units - 1) / run;  // the runs that have parts of it
      if (last_to_arrive(P, b0, (int)(b1 - b0 + 1)))
        join_many<TYPE, D, kChunkRows, kChunkThreads / 64>(A, it, of, rows, b0, (int)(b1 - b0 + 1), P.floats);
    }
  }
}

// The row kernel's parts where an item has many, which one block would be long
// in adding up (4 users of 131072 tokens, 64 parts an item: 92 us instead of
// 61).  A block takes one cut between runs; the cuts within one item share its
// elements, 64 a block, and its wavefronts share the parts.
constexpr int kJoinWaves = 8;
template <int TYPE, int D>
__global__ __launch_bounds__(64 * kJoinWaves) void k_join(AttendArgs A, Share share, int blocks, const float *floats) {
  constexpr int R = kRows;
  extern __shared__ uint32_t pre[];
  __shared__ float lm[kJoinWaves][64], ll[kJoinWaves][64], lo[kJoinWaves][64];
  const int group = A.n_q_heads / A.c.n_heads;
  const uint32_t total = list_units<64 * kJoinWaves, R>(A, group, share, pre), run = run_length(total, blocks, share);
  const uint32_t cut = (blockIdx.x + 1) * run;
  if (cut >= total) return;
  const Item it = item_at<R>(A, group, share, pre, cut);
  if (it.start == cut || stays_whole(it.units, run)) return;
  const uint32_t b0 = it.start / run, b1 = (it.start + it.units - 1) / run;  // the runs that have parts of it
  const int parts = (int)(b1 - b0 + 1), rows = min(R, it.q.n * group - it.r0);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Rows of(it.r0, group, A.per_group);
  for (int e = (int)(blockIdx.x - b0) * 64 + lane; e - lane < rows * D; e += (parts - 1) * 64) {  // rows * D is a multiple of 64
    const int i = e / D, d = e % D;
    float M = kFloor, sum = 0.0f, out = 0.0f;
#pragma unroll 8
    for (int p = wave; p < parts; p += kJoinWaves) {
      const float *const f = floats + part_index(b0 + p, p == 0) * part_floats(R, D);
      const float m = f[2 * i], l = f[2 * i + 1], v = f[2 * R + i * D + d];
      const float m_new = fmaxf(M, m);
      const float keep = __builtin_amdgcn_exp2f(M - m_new), add = __builtin_amdgcn_exp2f(m - m_new);
      sum = sum * keep + l * add;
      out = out * keep + v * add;
      M = m_new;
    }
    lm[wave][lane] = M;
    ll[wave][lane] = sum;
    lo[wave][lane] = out;
    __syncthreads();
    if (wave == 0) {
      for (int w = 1; w < kJoinWaves; ++w) M = fmaxf(M, lm[w][lane]);
      sum = out = 0.0f;
      for (int w = 0; w < kJoinWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(lm[w][lane] - M);
        sum += f * ll[w][lane];
        out += f * lo[w][lane];
      }
      const int2 at = of(i);
      store_value<TYPE>(A.out, ((int64_t)(it.q.q0 + at.x) * A.n_q_heads + it.h * group + at.y) * D + d,
                        sum == 0.0f ? 0.0f : out / sum);
    }
    __syncthreads();
  }
}

__global__ void k_check_attention(AttendArgs A, int32_t *flag) {
  const int s = blockIdx.x;
  const int q0 = A.cu_q[s], q1 = A.cu_q[s + 1], length = A.ctx_lens[s];
  if (threadIdx.x == 0) {
    if (q0 < 0 || q1 < q0 || q1 > A.n_tokens || (s == 0 && q0 != 0) ||
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

// A number that no other call of the process has; the start differs from process
// to process (a clock and where the program lies; nothing here may throw).
unsigned long long next_call() {
  static std::atomic<unsigned long long> number{
      (unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() * 0x9e3779b97f4a7c15ull ^
      (unsigned long long)(uintptr_t)&next_call};
  unsigned long long n;
  do n = ++number << 12;
  while (n == 0);
  return n;
}

// From what the host knows, at most: the units of an item.
int64_t most_units(const AttendArgs &A) {
  int64_t tiles = (A.table_width << A.c.page_shift) / kTile;
  if (A.window) tiles = std::min(tiles, ((int64_t)A.window + A.max_q) / kTile);
  return tiles + kItemUnits;
}

// Whether sequences of many rows go to the chunk kernel: from so many units of 16
// rows, e, on, earlier where items are short, as parts of 256 rows are costly to
// add.  Neither kernel's time follows from e alone (at the same e they are up to a
// factor of two apart from call to call); 13000 and 45000 are what parts the calls
// measured.  (us, chunk kernel and row kernel.  Up to 16 tiles: 310 tokens of 96
// heads in a window of 100, e = 14880, 32.5 and 32.9; 2 x 816 in one of 100,
// 21216, 30 and 41.  Longer: 147 tokens of 23 users over up to 1277, 16180, 42 and
// 22; one of 1095 over 1878, 32880, 100 and 73; 58 tokens of 20 users in a window
// of 1000, 45696, 86 and 109; 4 x 1704 over 1747, 93744, 53 and 100; 2 x 2048 over
// 8192, 40 heads, 680 and 1716.)  Both counts are upper bounds, from the table's
// width.  Of the tokens one a sequence is left out: in a
// step of many users and one prompt they are those that no chunk has (120 users,
// 79 tokens of 24 heads over 3869 among them: 65 us, by the chunk kernel 383).
bool takes_chunks(const AttendArgs &A, int kernel) {
  if (kernel) return kernel == 2;
  const int64_t group = A.n_q_heads / A.c.n_heads, tiles = most_units(A) - kItemUnits;
  const int64_t row_tiles = ((int64_t)std::max(0, A.n_tokens - A.n_seqs) * group / kRows + 1) * A.c.n_heads;
  return A.max_q * group >= kChunkLeast && row_tiles * std::max<int64_t>(tiles, kItemUnits) >= (tiles <= 16 ? 13000 : 45000);
}

template <int TYPE, int D, bool ONE>
hipError_t attend_as(const AttendArgs &A, int kernel, void *ws, hipStream_t s) {
  const size_t lds = sizeof(uint32_t) * A.n_seqs;
  const int64_t group = A.n_q_heads / A.c.n_heads, most_rows = A.max_q * group;
  const int everything = 0x7fffffff;
  const int64_t tiles = most_units(A);
  const bool chunks = takes_chunks(A, kernel);
  Parts P{(unsigned long long *)ws, (float *)((unsigned long long *)ws + kRowBlocks), 0};
  if (chunks) {
    // Alone where no sequence has few rows if the others have max_q tokens each and
    // all rows are someone's.  It takes any that has few all the same: lengths are
    // the device's, and a buffer may hold more rows than the sequences.
    const bool alone = kernel == 2 || A.n_seqs == 1 || (A.n_tokens - (A.n_seqs - 1) * (int64_t)A.max_q) * group >= kChunkLeast;
    const Share many{8, alone ? 1 : kChunkLeast, everything, 0};
    P.call = next_call();
    k_attend_chunk<TYPE, D, ONE><<<kChunkBlocks, kChunkThreads, lds, s>>>(A, many, P);
    if (alone) return hipGetLastError();
  }
  // about what there is: a sequence has a token at least
  const int64_t likely = ((int64_t)A.n_seqs * ((group + kRows - 1) / kRows) + std::max(0, A.n_tokens - A.n_seqs) * group / kRows) * A.c.n_heads;
  // Two blocks a CU of four wavefronts, or where there are fewer items than CUs
  // one of eight, which have half the tiles each before the parts are joined (but
  // not where a CU's share is a few tiles, one for each of the four).
  // (us a call, four and eight: 4 users of 1000 tokens and 8 heads 14.6 and
  // 11.8, 64 of 1000 and one head 15.3 and 12.0, 4 of 4000 and one head 19.8 and
  // 16.5, one of 1000 and one head 10.3 and 10.6; 32 of 4000 and 8 heads, 256
  // items, 27.1 and 29.1, 64 of 512 to 8192 73.5 and 94.7.)
  const auto rows = [&](auto waves_of) {
    constexpr int WAVES = decltype(waves_of)::value, BLOCKS = row_blocks(WAVES);
    // Where runs of 4, 8 or 16 units are enough for every item to be cut on its
    // own, they are (us a call, cut evenly and so: 4 users of 4000 tokens and one
    // head 16.4 and 12.4, 8 heads 20.3 and 16.4, 64 of 4000 and one head 23.7 and
    // 19.4; with lengths of 1000 to 16000 16 users of one head 21.1 and 25.1, 32 of
    // up to 8000 20.2 and 18.2).  Longer runs are cut evenly, as lengths differ.
    Share few{4, 1, chunks ? kChunkLeast : everything, 0};
    for (int run = 4; run <= 16; run *= 2)
      if (few.round == 0 && likely * ((tiles - kItemUnits + run - 1) / run) <= BLOCKS) {
        few.least = run;
        few.round = run - 1;
      }
    // parts of an item: by the length of its context, or by its share of the blocks
    const int64_t items = std::max<int64_t>(1, (int64_t)A.n_seqs * A.c.n_heads * ((std::min<int64_t>(most_rows, kChunkLeast) + kRows - 1) / kRows));
    const bool few_parts = std::min((tiles - kItemUnits) / few.least, 2 * BLOCKS / items) < 12;
    P.call = few_parts ? next_call() : 0;
    k_attend_rows<TYPE, D, WAVES, ONE><<<BLOCKS, 64 * WAVES, lds, s>>>(A, few, P);
    if (!few_parts) k_join<TYPE, D><<<BLOCKS - 1, 64 * kJoinWaves, lds, s>>>(A, few, BLOCKS, P.floats);
    return hipGetLastError();
  };
  const bool wide = likely <= 224 && likely * ((tiles - kItemUnits + 3) / 4) > 64;
  return wide ? rows(std::integral_constant<int, 8>{}) : rows(std::integral_constant<int, 4>{});
}

}  // namespace

size_t attention_workspace(const Cache &c, int32_t, int64_t, int32_t) {
  // a counter a run and at most two parts; the kernels run one after the other
  return kRowBlocks * sizeof(unsigned long long) +
         2 * sizeof(float) * std::max(kRowBlocks * part_floats(kRows, c.head_dim), kChunkBlocks * part_floats(kChunkRows, c.head_dim));
}

bool attention_fits(const AttendArgs &A, int kernel) {
  const int64_t group = A.n_q_heads / A.c.n_heads, rows = (int64_t)A.n_tokens * group;
  const auto fits = [&](int64_t row_tiles) { return row_tiles <= 0x7fffffff / A.c.n_heads / (most_units(A) + 16); };
  if (!takes_chunks(A, kernel)) return fits(rows / kRows + A.n_seqs);
  return fits(rows / kChunkRows + A.n_seqs) && fits((int64_t)A.n_seqs * (kChunkLeast / kRows));
}

template <int TYPE>
static hipError_t attend_of(const AttendArgs &A, int kernel, void *ws, hipStream_t s) {
  if (A.c.page_shift == 6) return A.c.head_dim == 64 ? attend_as<TYPE, 64, true>(A, kernel, ws, s) : attend_as<TYPE, 128, true>(A, kernel, ws, s);
  return A.c.head_dim == 64 ? attend_as<TYPE, 64, false>(A, kernel, ws, s) : attend_as<TYPE, 128, false>(A, kernel, ws, s);
}

hipError_t launch_cache_attention(const AttendArgs &A, int kernel, void *ws, hipStream_t s) {
  return A.type == kF16 ? attend_of<kF16>(A, kernel, ws, s) : attend_of<kBF16>(A, kernel, ws, s);
}

hipError_t launch_check_attention(const AttendArgs &A, int32_t *flag, hipStream_t s) {
  k_check_attention<<<A.n_seqs, 64, 0, s>>>(A, flag);
  return hipGetLastError();
}

}  // namespace fs
