// fs_project.hip -- projections with what stands before and behind them in a
// decoder layer: the rows' RMS norm in front of the quantisation; an activation
// and the residual stream behind the product, or the product of the activated
// gate and the value, while the sums are in registers.
//
// Bounds: up to a few hundred rows the weights' bytes, then the matrix units.
// Against the separate calls a layer saves the norms', the activation's and the
// sums' launches and their passes over the rows, and a gated block's gates and
// values are never stored: a decoder layer of 5120 channels takes 43 us instead of 63
// for one token on a TP8 shard (of 80 layers, a cache of 1152 tokens).
//
// Measured, weights from memory: one row of 5120 x 5120 7.1 us (3.7 TB/s, the
// weights' bytes' time 5.1: a block's chain of the row's loads, its codes and ten stages of
// weights, in 160 blocks on 256 CUs), normed and gated by 2 x 2560 8.1; 64 rows by 2 x
// 20480, K = 5120, 57.5 (5 of them the codes' launch, then 4.0 TB/s: a stage's chain of
// barrier, LDS and products keeps its loads from filling the memory; deeper rings,
// wider tiles and two blocks a CU took 57 to 61); 4096 rows of the same 735 to 765 by
// the card (2.3 PO/s).
#include "fs_product.h"

namespace fs {
namespace {

constexpr int kAnyType = -1;  // the output's type is looked at when a tile is stored

template <Finish FINISH>
bool few_finished(const QuantizeArgs &X, const MatmulArgs &A, hipStream_t s, hipError_t *e) {
  return X.normed ? few_of<kAnyType, FINISH, true>(X, A, s, e) : few_of<kAnyType, FINISH, false>(X, A, s, e);
}

}  // namespace

bool launch_project_few(const QuantizeArgs &X, const MatmulArgs &A, bool gated, hipStream_t s, hipError_t *e) {
  if (!few_rows(X, A)) return false;
  if (gated && A.N * A.w_stride > (int64_t)1 << 31) return false;  // both rows of a channel: in 32 bits from the first on
  return gated ? few_finished<kGated>(X, A, s, e) : few_finished<kFinished>(X, A, s, e);
}

PartsRoom parts_room(int64_t M, int64_t w_rows, int64_t K) {
  if (M == 0 || w_rows == 0 || K < 2 * kLeastPart) return {};
  // Which tiles are left over, and so what a cut needs, goes up and down with the rows.
  // Of a few rows the most that as many or fewer need (all tiles' heights are multiples of
  // 16), of more what the largest tile could.
  int64_t sums = 0;
  if (M > 128) {
    for (const Tile &t : kTiles) sums = std::max<int64_t>(sums, kMostParts * t.bm * t.bn * 4);
  } else {
    for (int64_t m = 16; m - 16 < M; m += 16) sums = std::max(sums, choose((int32_t)m, (int32_t)w_rows, (int32_t)K).bytes());
  }
  return {(size_t)kMostParts * 4, (size_t)sums};
}

void plan_project(int64_t M, int64_t w_rows, int64_t K, void *counts, void *sums, QuantizeArgs *rows, MatmulArgs *product) {
  const Choice c = choose((int32_t)M, (int32_t)w_rows, (int32_t)K);
  product->tile = c.tile;
  product->whole = (int32_t)c.whole;  // see project_fits
  product->parts = c.parts;
  product->arrived = (int32_t *)counts;
  product->partials = (int32_t *)sums;
  rows->zero = (int32_t *)counts;
  rows->n_zero = (int32_t)c.slots();
}

bool project_fits(int64_t M, int64_t w_rows, int64_t K) {
  const Choice c = choose((int32_t)M, (int32_t)w_rows, (int32_t)K);
  return 8 * (c.whole + c.rest * c.parts) <= kMostBlocks;
}

hipError_t launch_quantize_normed(const QuantizeArgs &A, hipStream_t s) {
  return A.type == kF32   ? quantize_of<kF32, true>(A, s)
         : A.type == kF16 ? quantize_of<kF16, true>(A, s)
                          : quantize_of<kBF16, true>(A, s);
}

hipError_t launch_project(const MatmulArgs &A, bool gated, hipStream_t s) {
  return gated ? matmul_of<kAnyType, kGated>(A, s) : matmul_of<kAnyType, kFinished>(A, s);
}

}  // namespace fs
