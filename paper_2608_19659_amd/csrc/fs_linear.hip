// fs_linear.hip -- projections in 8-bit integers: rows of activations to
// codes with a scale a row, and the product of codes with weights that have a
// scale an output channel.
//
// y[m][n] = (sum_k a[m][k] w[n][k]) * a_scale[m] * w_scale[n] + bias[n].
// The sum is exact in 32-bit integers whatever the order, so tiles, splits
// and instructions are free to choose and every variant gives the same bits.
#include "fs_serving.h"

namespace fs {
namespace {

// The largest |x| of a block's values by their bit patterns: a NaN is larger
// than an infinity, so neither is lost in the maximum.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

template <int THREADS>
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t *lds) {
  for (int o = 32; o; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  if constexpr (THREADS > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int i = 1; i < THREADS / 64; ++i) v = max(v, lds[i]);
  }
  return v;
}

// One block a row.
template <int TYPE>
__global__ __launch_bounds__(256) void k_quantize_rows(QuantizeArgs A) {
  __shared__ uint32_t lds[4];
  const int64_t row = blockIdx.x;
  const int64_t at = row * A.x_stride;
  uint32_t most = 0;
  for (int c = threadIdx.x; c < A.cols; c += 256) most = max(most, magnitude(load_value<TYPE>(A.x, at + c)));
  const float a = __uint_as_float(block_max<256>(most, lds));
  const bool zero = a < kTiny;
  const float inverse = zero ? 0.0f : 127.0f / a;
  int8_t *out = A.codes + row * A.code_stride;
  for (int c = threadIdx.x; c < A.cols; c += 256) {
    const float x = load_value<TYPE>(A.x, at + c);
    out[c] = zero ? (int8_t)0 : (int8_t)(int)rintf(x * inverse);
  }
  if (threadIdx.x == 0) A.scale[row] = zero ? 0.0f : a / 127.0f;
}

// 16 codes of a row from column k on, zeros beyond its end.  Rows may start
// anywhere: the load is one of 16 bytes at any alignment.
__device__ __forceinline__ int4v codes16(const int8_t *row, int k, int K) {
  int4v v = {0, 0, 0, 0};
  if (k + 16 <= K) {
    __builtin_memcpy(&v, row + k, 16);
  } else {
    for (int i = 0; i < 16; ++i)
      if (k + i < K) v[i >> 2] |= (int)((uint32_t)(uint8_t)row[k + i] << (8 * (i & 3)));
  }
  return v;
}

template <int TYPE>
__device__ __forceinline__ void store_products(const MatmulArgs &A, int m, int n, int4v acc, float sa) {
  // four neighbouring channels of one token
  const int64_t at = (int64_t)m * A.out_stride + n;
  for (int i = 0; i < 4; ++i)
    if (n + i < A.N) {
      float y = (float)acc[i] * sa * A.w_scale[n + i];
      if (A.bias) y += A.bias[n + i];
      store_value<TYPE>(A.out, at + i, y);
    }
}

// Tiles of 64 tokens x 64 channels, 128 inner elements at a time through LDS.
// The weights are the instruction's first operand, so a lane's four results
// are neighbours in a row of the output.  LDS rows of eight 16-byte chunks,
// chunk c of row r at place c ^ ((r >> 1) & 7): the 16 rows that a quarter of
// a wavefront reads fall on all 64 banks.
template <int TYPE>
__global__ __launch_bounds__(256) void k_matmul_tile(MatmulArgs A) {
  __shared__ int4v la[64 * 8], lw[64 * 8];
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = (wave & 1) * 32, wn = (wave >> 1) * 32;
  int4v acc[2][2] = {};
  for (int k0 = 0; k0 < A.K; k0 += 128) {
    for (int i = 0; i < 2; ++i) {
      const int chunk = threadIdx.x + 256 * i, r = chunk >> 3, c = chunk & 7;
      const int to = r * 8 + (c ^ ((r >> 1) & 7)), k = k0 + c * 16;
      la[to] = codes16(A.a + (int64_t)min(m0 + r, A.M - 1) * A.a_stride, k, A.K);
      lw[to] = codes16(A.w + (int64_t)min(n0 + r, A.N - 1) * A.w_stride, k, A.K);
    }
    __syncthreads();
    for (int kk = 0; kk < 2; ++kk) {
      int4v fa[2], fw[2];
      for (int i = 0; i < 2; ++i) {
        const int c = kk * 4 + (lane >> 4), ra = wm + i * 16 + (lane & 15), rw = wn + i * 16 + (lane & 15);
        fa[i] = la[ra * 8 + (c ^ ((ra >> 1) & 7))];
        fw[i] = lw[rw * 8 + (c ^ ((rw >> 1) & 7))];
      }
      for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[j], fa[i], acc[i][j], 0, 0, 0);
    }
    __syncthreads();
  }
  for (int i = 0; i < 2; ++i) {
    const int m = m0 + wm + i * 16 + (lane & 15);
    if (m >= A.M) continue;
    const float sa = A.a_scale[m];
    for (int j = 0; j < 2; ++j) store_products<TYPE>(A, m, n0 + wn + j * 16 + (lane >> 4) * 4, acc[i][j], sa);
  }
}

}  // namespace

hipError_t launch_quantize_rows(const QuantizeArgs &A, hipStream_t s) {
  if (A.type == kF32) k_quantize_rows<kF32><<<A.rows, 256, 0, s>>>(A);
  else if (A.type == kF16) k_quantize_rows<kF16><<<A.rows, 256, 0, s>>>(A);
  else k_quantize_rows<kBF16><<<A.rows, 256, 0, s>>>(A);
  return hipGetLastError();
}

size_t matmul_workspace(int32_t, int32_t, int32_t) { return 0; }

hipError_t launch_scaled_matmul(const MatmulArgs &A, void *, hipStream_t s) {
  const dim3 grid((A.N + 63) / 64, (A.M + 63) / 64);
  if (A.out_type == kF32) k_matmul_tile<kF32><<<grid, 256, 0, s>>>(A);
  else if (A.out_type == kF16) k_matmul_tile<kF16><<<grid, 256, 0, s>>>(A);
  else k_matmul_tile<kBF16><<<grid, 256, 0, s>>>(A);
  return hipGetLastError();
}

}  // namespace fs
