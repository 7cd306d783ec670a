// The matrix-core products of bf16 operands (and of fp32 ones in three bf16 parts), and the
// choice of their tiles and splits.
#include "layers_mm.h"

namespace pointid {

ProductPlan plan_product(Form form, int64_t rows, int64_t cols, int halves, int64_t inner, int terms, int cus) {
  ProductPlan p;
  const int64_t its = (inner + mm::kBK - 1) / mm::kBK * terms;
  auto tiles = [&](int t) {
    const int64_t n = kTileN[t] / halves;
    return ((rows + kTileM[t] - 1) / kTileM[t]) * ((cols + n - 1) / n);
  };
  p.tile = 0;
  while (p.tile < kTiles - 1 && tiles(p.tile) < cus) ++p.tile;
  // fewer tiles than CUs: the sum is split, each part at least 4 stages long
  const int64_t t = tiles(p.tile);
  int64_t s = t < cus ? cus / t : 1;
  if (s > its / 4) s = its / 4;
  p.splits = (int)(s < 1 ? 1 : s);
  return p;
}

hipError_t launch_product_bf16(Form form, const ProductPlan& plan, ProductArgs a, hipStream_t stream) {
  return mm::launch<false>(form, plan, a, stream);
}

}  // namespace pointid
