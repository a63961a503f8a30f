// fs_linear.hip -- projections in 8-bit integers: the launchers of the row
// quantisation and of the product with scales and a bias.
#include "fs_product.h"

namespace fs {

bool launch_linear_few(const QuantizeArgs &X, const MatmulArgs &A, hipStream_t s, hipError_t *e) {
  if (!few_rows(X, A)) return false;
  return A.out_type == kF32 ? few_of<kF32, kScaled, false>(X, A, s, e)
         : A.out_type == kF16 ? few_of<kF16, kScaled, false>(X, A, s, e)
                              : few_of<kBF16, kScaled, false>(X, A, s, e);
}

hipError_t launch_quantize_rows(const QuantizeArgs &A, hipStream_t s) {
  return A.type == kF32   ? quantize_of<kF32, false>(A, s)
         : A.type == kF16 ? quantize_of<kF16, false>(A, s)
                          : quantize_of<kBF16, false>(A, s);
}

bool matmul_fits(int32_t M, int32_t N, int32_t K) {
  const Tile &t = kTiles[best_tile(M, N, K)];
  return ((int64_t)(M - 1) / t.bm + 1) * ((N - 1) / t.bn + 1) <= kMostBlocks;
}

hipError_t launch_scaled_matmul(const MatmulArgs &A, hipStream_t s) {
  return A.out_type == kF32   ? matmul_of<kF32, kScaled>(A, s)
         : A.out_type == kF16 ? matmul_of<kF16, kScaled>(A, s)
                              : matmul_of<kBF16, kScaled>(A, s);
}

}  // namespace fs
