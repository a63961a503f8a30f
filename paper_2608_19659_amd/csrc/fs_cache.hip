// fs_cache.hip -- the paged 8-bit key/value cache: appending a step's tokens
// with the position rotation applied on the way, and reading values back.
#include <algorithm>

#include "fs_serving.h"

namespace fs {
namespace {

__device__ int32_t g_flag[4];  // FS_VALIDATE=1: what the checks counted

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ int64_t n_slots(const Cache &c) { return (int64_t)c.n_pages << c.page_shift; }

// The code of a value under the inverse of its scale.
__device__ __forceinline__ int code_of(float x, float inverse) {
  return (int)fminf(fmaxf(rintf(x * inverse), -127.0f), 127.0f);
}

// Element d of a rotated row: x' = x cos -+ partner sin, each rounded.
template <int TYPE>
__device__ __forceinline__ float rotated(const AppendArgs &A, const void *x, int64_t row, int d, int position) {
  const float v = load_value<TYPE>(x, row + d);
  if (d >= 2 * A.half) return v;
  const bool low = d < A.half;
  const int i = low ? d : d - A.half;
  const int64_t at = (int64_t)position * A.half + i;
  const float c = A.cosines[at], s = A.sines[at], w = load_value<TYPE>(x, row + (low ? d + A.half : i));
  return low ? v * c - w * s : v * c + w * s;
}

__device__ __forceinline__ int position_of(const AppendArgs &A, int t) {
  return A.half ? min(max(A.positions[t], 0), A.n_positions - 1) : 0;
}

// One page's keys (or values) of one head: the new tokens in binary32 in LDS,
// their largest magnitude, the page's new scale, then the codes.  The codes
// held are read and written only where the scale grows.
template <int TYPE, int D, bool VALUES>
__device__ void append_page(const AppendArgs &A, int t, int slot, int head, float *lds, uint32_t *most) {
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
  if (threadIdx.x == 0) *most = 0;
  __syncthreads();
  uint32_t m = 0;
  for (int e = threadIdx.x; e < n * D; e += 256) {
    const int j = e / D, d = e % D;
    float x;
    if constexpr (VALUES) x = load_value<TYPE>(A.v, (t + j) * A.v_stride + head * D + d);
    else x = rotated<TYPE>(A, A.k, (t + j) * A.k_stride + head * D, d, position_of(A, t + j));
    lds[e] = x;
    m = max(m, magnitude(x));
  }
  for (int o = 32; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
  if (lane == 0) atomicMax(most, m);
  __syncthreads();
  const float a = __uint_as_float(*most), made = a < kTiny ? 0.0f : a / 127.0f;
  const float now = old >= made || old != old ? old : made;  // a NaN on either side stays
  const bool grew = first && !(now == old);
  const float inverse = now > 0.0f ? 1.0f / now : 0.0f, ratio = now > 0.0f ? old / now : 0.0f;
  if constexpr (VALUES) {  // a thread owns 16 tokens of one element
    const int g0 = grew ? 0 : first >> 4, g1 = (first + n - 1) >> 4, ng = g1 - g0 + 1;
    for (int e = threadIdx.x; e < D * ng; e += 256) {
      const int d = e / ng, g = g0 + e % ng;
      int4v *const p = (int4v *)(codes + d * PS + g * 16);
      int4v row = *p;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = g * 16 + i, shift = 8 * (i & 3);
        const int held = (int)(int8_t)(row[i >> 2] >> shift);
        int code = held;
        if (at >= first && at < first + n) code = code_of(lds[(at - first) * D + d], inverse);
        else if (grew && at < first) code = (int)rintf((float)held * ratio);
        row[i >> 2] = (row[i >> 2] & ~(0xff << shift)) | ((code & 0xff) << shift);
      }
      *p = row;
    }
  } else {
    if (grew)
      for (int e = threadIdx.x; e < first * D; e += 256) codes[e] = (int8_t)(int)rintf((float)codes[e] * ratio);
    for (int e = threadIdx.x; e < n * D; e += 256) codes[first * D + e] = (int8_t)code_of(lds[e], inverse);
  }
  if (threadIdx.x == 0) *scale = now;
  __syncthreads();
}

// blockIdx.x: a run of `span` tokens; blockIdx.y: the keys and the values of
// each cache head, then blocks of query heads.
template <int TYPE, int D>
__global__ __launch_bounds__(256) void k_append(AppendArgs A, int span) {
  extern __shared__ float lds[];
  __shared__ uint32_t most;
  const int t0 = blockIdx.x * span, t1 = min(t0 + span, A.n_tokens), PS = 1 << A.c.page_shift;
  const int first_q = 2 * A.c.n_heads, part = blockIdx.y;
  if (part < first_q) {
    for (int t = t0; t < t1; ++t) {
      const int slot = A.slots[t];
      if (slot < 0 || slot >= n_slots(A.c)) continue;
      // not the page's first new token: the block of the one before does it
      if (t > 0 && (slot & (PS - 1)) && A.slots[t - 1] == slot - 1) continue;
      if (part & 1) append_page<TYPE, D, true>(A, t, slot, part >> 1, lds, &most);
      else append_page<TYPE, D, false>(A, t, slot, part >> 1, lds, &most);
    }
    return;
  }
  const int width = A.n_q_heads * D, step = (gridDim.y - first_q) * 256;
  for (int t = t0; t < t1; ++t) {
    const int position = position_of(A, t);
    for (int e = (part - first_q) * 256 + threadIdx.x; e < width; e += step)
      store_value<TYPE>(A.q_out, (int64_t)t * width + e, rotated<TYPE>(A, A.q, t * A.q_stride + e / D * D, e % D, position));
  }
}

template <int TYPE, int D>
__global__ __launch_bounds__(256) void k_read(ReadArgs A) {
  const Cache &c = A.c;
  const int PS = 1 << c.page_shift;
  const int t0 = blockIdx.x * 16, head = blockIdx.y;
  for (int e = threadIdx.x; e < 16 * D; e += 256) {
    const int t = t0 + e / D, d = e % D;
    if (t >= A.n_tokens) break;
    const int slot = A.slots[t];
    const bool in = slot >= 0 && slot < n_slots(c);
    const int64_t block = (int64_t)((in ? slot : 0) >> c.page_shift) * c.n_heads + head;
    const int place = (in ? slot : 0) & (PS - 1);
    const int64_t to = ((int64_t)t * c.n_heads + head) * D + d;
    if (A.k_out) store_value<TYPE>(A.k_out, to, in ? (float)c.k[(block * PS + place) * D + d] * c.k_scale[block] : 0.0f);
    if (A.v_out) store_value<TYPE>(A.v_out, to, in ? (float)c.v[(block * D + d) * PS + place] * c.v_scale[block] : 0.0f);
  }
}

__global__ void k_clear(int32_t *flag) {
  if (threadIdx.x < 4) flag[threadIdx.x] = 0;
}

__global__ void k_check_slots(Cache c, const int32_t *slots, const int32_t *positions, int32_t n_positions, int32_t n,
                              int appending, int32_t *flag) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= n) return;
  const int slot = slots[t];
  if (slot >= n_slots(c) || (slot < 0 && !appending)) atomicAdd(&flag[0], 1);
  if (positions && (positions[t] < 0 || positions[t] >= n_positions)) atomicAdd(&flag[1], 1);
  if (appending && t > 0 && slot >= 0 && slots[t - 1] >= 0) {
    const int before = slots[t - 1];
    if ((before >> c.page_shift) == (slot >> c.page_shift) && before != slot - 1) atomicAdd(&flag[2], 1);
  }
}

}  // namespace

hipError_t flag_address(int32_t **flag) { return hipGetSymbolAddress((void **)flag, HIP_SYMBOL(g_flag)); }

hipError_t launch_clear_flag(int32_t *flag, hipStream_t s) {
  k_clear<<<1, 64, 0, s>>>(flag);
  return hipGetLastError();
}

hipError_t launch_check_slots(const Cache &c, const int32_t *slots, const int32_t *positions, int32_t n_positions,
                              int32_t n_tokens, int appending, int32_t *flag, hipStream_t s) {
  k_check_slots<<<(n_tokens + 255) / 256, 256, 0, s>>>(c, slots, positions, n_positions, n_tokens, appending, flag);
  return hipGetLastError();
}

template <int TYPE, int D>
static hipError_t append_as(const AppendArgs &A, hipStream_t s) {
  const int span = A.n_tokens <= 2048 ? 1 : 16;
  const int q_blocks = A.q ? std::min(16, (A.n_q_heads * D + 255) / 256) : 0;
  const dim3 grid((A.n_tokens + span - 1) / span, 2 * A.c.n_heads + q_blocks);
  k_append<TYPE, D><<<grid, 256, sizeof(float) * (D << A.c.page_shift), s>>>(A, span);
  return hipGetLastError();
}

template <int TYPE>
static hipError_t append_of(const AppendArgs &A, hipStream_t s) {
  return A.c.head_dim == 64 ? append_as<TYPE, 64>(A, s) : append_as<TYPE, 128>(A, s);
}

hipError_t launch_cache_append(const AppendArgs &A, hipStream_t s) {
  return A.type == kF32 ? append_of<kF32>(A, s) : A.type == kF16 ? append_of<kF16>(A, s) : append_of<kBF16>(A, s);
}

template <int TYPE>
static hipError_t read_of(const ReadArgs &A, hipStream_t s) {
  const dim3 grid((A.n_tokens + 15) / 16, A.c.n_heads);
  if (A.c.head_dim == 64) k_read<TYPE, 64><<<grid, 256, 0, s>>>(A);
  else k_read<TYPE, 128><<<grid, 256, 0, s>>>(A);
  return hipGetLastError();
}

hipError_t launch_cache_read(const ReadArgs &A, hipStream_t s) {
  return A.type == kF32 ? read_of<kF32>(A, s) : A.type == kF16 ? read_of<kF16>(A, s) : read_of<kBF16>(A, s);
}

}  // namespace fs
