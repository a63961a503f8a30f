// fs_serving.h -- the serving operators' launchers (host) and the element
// conversions their kernels share.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace fs {

enum Dtype : int32_t { kF32 = 0, kF16 = 1, kBF16 = 2 };

// A row or block whose largest magnitude is below this counts as zero.
constexpr float kTiny = 0x1p-100f;
// A page scale below this stands for a page of zeros.
constexpr float kZeroScale = 0x1p-110f;

struct QuantizeArgs {
  const void *x;
  int8_t *codes;
  float *scale;
  int64_t x_stride, code_stride;
  int32_t rows, cols, type;
  int32_t normed;     // the rows' RMS norm first:
  const float *gain;  // factor of each column, NULL for ones
  float eps;
  int32_t *zero;  // cleared on the way
  int32_t n_zero;
};
hipError_t launch_quantize_rows(const QuantizeArgs &A, hipStream_t s);

enum Activation : int32_t { kNoActivation = 0, kRelu = 1, kGelu = 2, kGeluTanh = 3, kSilu = 4 };

// A launch has fewer than 2^32 threads along its grid's first dimension: blocks
// of up to 512 threads, in multiples of eight, are at most this many.
constexpr int64_t kMostBlocks = (1 << 23) - 8;

struct MatmulArgs {
  const int8_t *a, *w;
  const float *a_scale, *w_scale, *bias;
  void *out;
  int64_t a_stride, w_stride, out_stride;
  int32_t M, N, K, out_type;
  int32_t a_padded;  // rows of a may be read (not their values used) to the next multiple of 16
  // launch_project only:
  int32_t activation;
  const void *residual;  // of out's type, or NULL; may be out
  int64_t residual_stride;
  int32_t tile, whole, parts;  // set by plan_project
  int32_t *arrived, *partials;
};
// Whether the product's tiles are few enough for one launch.
bool matmul_fits(int32_t M, int32_t N, int32_t K);
hipError_t launch_scaled_matmul(const MatmulArgs &A, hipStream_t s);

// Both steps in one launch where there are few rows (codes and scales stay
// unset); false: not for this call, nothing done.
bool launch_linear_few(const QuantizeArgs &X, const MatmulArgs &A, hipStream_t s, hipError_t *e);

// The same with an RMS norm before and an activation and a residual behind, or
// gated: w has 2 N rows, the gates' and then the values'.
hipError_t launch_quantize_normed(const QuantizeArgs &A, hipStream_t s);
// Bytes for the counts and the parts' sums of products of w_rows weight rows, of M
// rows and of fewer.
struct PartsRoom {
  size_t counts, sums;
};
PartsRoom parts_room(int64_t M, int64_t w_rows, int64_t K);
// Gives `rows` and `product` these places and how the product is cut.
void plan_project(int64_t M, int64_t w_rows, int64_t K, void *counts, void *sums, QuantizeArgs *rows, MatmulArgs *product);
bool project_fits(int64_t M, int64_t w_rows, int64_t K);
hipError_t launch_project(const MatmulArgs &A, bool gated, hipStream_t s);
bool launch_project_few(const QuantizeArgs &X, const MatmulArgs &A, bool gated, hipStream_t s, hipError_t *e);

struct Cache {
  int8_t *k, *v;
  float *k_scale, *v_scale;
  int32_t n_pages, n_heads, head_dim, page_shift;  // page size = 1 << page_shift
};

struct AppendArgs {
  Cache c;
  const void *k, *v, *q;
  void *q_out;
  const int32_t *slots, *positions;
  const float *cosines, *sines;
  int64_t k_stride, v_stride, q_stride;
  int32_t n_tokens, n_q_heads, type, n_positions, half;
};
hipError_t launch_cache_append(const AppendArgs &A, hipStream_t s);

struct ReadArgs {
  Cache c;
  const int32_t *slots;
  void *k_out, *v_out;
  int32_t n_tokens, type;
};
hipError_t launch_cache_read(const ReadArgs &A, hipStream_t s);

struct AttendArgs {
  Cache c;
  const void *q;
  void *out;
  const int32_t *cu_q, *ctx_lens, *table;
  int64_t q_stride, table_width;
  int32_t n_tokens, n_seqs, n_q_heads, max_q, window, type;
  float scale;
  uint32_t per_group;  // 2^32 / query heads of a group, rounded up (of no account for 1)
};
// `kernel`: 0 by size, 1 the kernel of 16 rows, 2 that of 256.
// Whether the call's units of work can be counted in 32 bits.
bool attention_fits(const AttendArgs &A, int kernel);
size_t attention_workspace(const Cache &c, int32_t n_q_heads, int64_t n_tokens, int32_t n_seqs);
hipError_t launch_cache_attention(const AttendArgs &A, int kernel, void *ws, hipStream_t s);

struct StateArgs {
  float *states;  // [n_states][n_heads][head_dim][head_dim]: keys' elements, then values'
  const void *q, *k, *v;
  void *out;
  const int32_t *cu_q, *ctx_lens, *index;
  const float *log_decay;
  float *local;  // workspace
  int64_t q_stride, k_stride, v_stride;
  int32_t n_states, n_heads, head_dim, n_q_heads, n_tokens, n_seqs, max_q, type;
  float scale;
  int32_t step_most, segment, n_places;  // set by the launcher
};
size_t state_workspace(int32_t n_heads, int32_t head_dim, int64_t n_tokens, int32_t n_seqs);
hipError_t launch_state_attention(const StateArgs &A, hipStream_t s);
hipError_t launch_check_state(const StateArgs &A, int32_t *flag, hipStream_t s);

// FS_VALIDATE=1: counts what is out of range into the validation words
// (flag_address) of the current device, which the caller cleared.
hipError_t flag_address(int32_t **flag);
hipError_t launch_clear_flag(int32_t *flag, hipStream_t s);
hipError_t launch_check_slots(const Cache &c, const int32_t *slots, const int32_t *positions, int32_t n_positions,
                              int32_t n_tokens, int appending, int32_t *flag, hipStream_t s);
hipError_t launch_check_attention(const AttendArgs &A, int32_t *flag, hipStream_t s);

#ifdef __HIPCC__
using half8 = _Float16 __attribute__((ext_vector_type(8)));
using float4v = float __attribute__((ext_vector_type(4)));
using float16v = float __attribute__((ext_vector_type(16)));
using int4v = int __attribute__((ext_vector_type(4)));

// 16 bytes from any address: the five words that hold them, shifted when they
// are there.  A load of 16 bytes off a word boundary takes the memory pipe
// many times as long.  Only words of which a byte is wanted are read.
struct Words {
  int4v first;
  uint32_t next, off;

  __device__ __forceinline__ void load(const void *p) {
    using int4w = int __attribute__((ext_vector_type(4), aligned(4)));
    using Word = const __attribute__((address_space(1))) uint32_t;
    off = (uint32_t)(uintptr_t)p & 3;
    Word *const w = (Word *)((uintptr_t)p & ~(uintptr_t)3);
    first = *(const __attribute__((address_space(1))) int4w *)w;
    next = w[off ? 4 : 3];
  }
  __device__ __forceinline__ void set(int4v v) {
    first = v;
    next = off = 0;
  }
  __device__ __forceinline__ int4v value() const {
    return int4v{(int)__builtin_amdgcn_alignbyte(first[1], first[0], off), (int)__builtin_amdgcn_alignbyte(first[2], first[1], off),
                 (int)__builtin_amdgcn_alignbyte(first[3], first[2], off), (int)__builtin_amdgcn_alignbyte(next, first[3], off)};
  }
};
__device__ __forceinline__ int4v load16(const void *p) {
  Words w;
  w.load(p);
  return w.value();
}

// Element types by their number: 2-byte types travel as raw 16-bit words.
__device__ __forceinline__ float bf16_value(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ uint16_t bf16_bits(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ float f16_value(uint16_t w) { return (float)__builtin_bit_cast(_Float16, w); }
__device__ __forceinline__ uint16_t f16_bits(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }

template <int TYPE>
__device__ __forceinline__ float load_value(const void *p, int64_t i) {
  if constexpr (TYPE == kF32) return ((const float *)p)[i];
  else if constexpr (TYPE == kF16) return f16_value(((const uint16_t *)p)[i]);
  else return bf16_value(((const uint16_t *)p)[i]);
}
template <int TYPE>
__device__ __forceinline__ void store_value(void *p, int64_t i, float v) {
  if constexpr (TYPE == kF32) ((float *)p)[i] = v;
  else if constexpr (TYPE == kF16) ((uint16_t *)p)[i] = f16_bits(v);
  else ((uint16_t *)p)[i] = bf16_bits(v);
}
// The 16-bit pattern of a value in a 2-byte type, and back.
template <int TYPE>
__device__ __forceinline__ uint16_t bits16(float v) {
  if constexpr (TYPE == kF16) return f16_bits(v);
  else return bf16_bits(v);
}
template <int TYPE>
__device__ __forceinline__ float value16(uint16_t w) {
  if constexpr (TYPE == kF16) return f16_value(w);
  else return bf16_value(w);
}
// Eight neighbouring elements from any place; `whole`: it is a multiple of 16
// bytes.
template <int TYPE>
__device__ __forceinline__ void load8(const void *x, int64_t at, bool whole, float (&v)[8]) {
  if constexpr (TYPE == kF32) {
    __builtin_memcpy(v, (const float *)x + at, 32);
  } else {
    const uint16_t *const p = (const uint16_t *)x + at;
    const int4v raw = whole ? *(const int4v *)p : load16(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = value16<TYPE>((uint16_t)(raw[i >> 1] >> 16 * (i & 1)));
  }
}
// Eight neighbouring elements to any place.
template <int TYPE>
__device__ __forceinline__ void store8(void *x, int64_t at, const float (&v)[8]) {
  if constexpr (TYPE == kF32) {
    __builtin_memcpy((float *)x + at, v, 32);
  } else {
    int4v raw;
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = (int)(bits16<TYPE>(v[2 * i]) | (uint32_t)bits16<TYPE>(v[2 * i + 1]) << 16);
    __builtin_memcpy((uint16_t *)x + at, &raw, 16);
  }
}
#endif

}  // namespace fs
