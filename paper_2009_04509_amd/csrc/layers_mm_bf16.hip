// The matrix-core products of bf16 operands (and of fp32 ones in three bf16 parts), and the
// choice of their tiles and splits.
#include "layers_mm.h"

#include <algorithm>
#include <cmath>

namespace pointid {

namespace {

// us of a tile shape, fitted to sweeps of tiles and splits over 23 products of all forms
// from 16 x 8192 x 8192 to 16384 x 1024 x 1024 (13 in fp32): a stage of 64 inner indices when
// `resident` blocks share a CU (each) and of a block alone, and a block's start and end.
// The choice by them is the fastest measured or within 3 % of it.
struct TileCost {
  double stage, alone, ends;
  int resident;
};
constexpr TileCost kCost[kTiles] = {{1.3, 1.3, 9.0, 1}, {0.57, 0.62, 3.4, 2}, {0.315, 0.435, 2.6, 3}};
constexpr TileCost kCost32[kTiles32] = {{4.47, 4.47, 2.5, 1}, {2.9, 2.9, 2.0, 1}, {1.56, 2.5, 1.9, 2}};

}  // namespace

// The tile and split that the costs above put first.  Large tiles read their operands fewer
// times (bf16 4096 x 1024 x 4096: 43 us in 256 x 256 tiles, 46 in 128 x 128, 55 in 64 x 128);
// small ones fill the CUs where there are few (2048^3: 29 in 64 x 128, 32 in 128 x 128, 44
// in split 256 x 256; its gated form 41 in 128 x 128, 55 in both others).
ProductPlan plan_product(bool f32, int64_t rows, int64_t cols, int halves, int64_t inner, int terms, int cus) {
  static constexpr int kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128};
  const double stages = (double)((inner + 63) / 64) * terms;
  const double part_mb = 8e-6 * (double)rows * (double)cols * halves;          // written and read
  ProductPlan best = {0, 1};
  double least = 1e300;
  for (int t = 0; t < (f32 ? kTiles32 : kTiles); ++t) {
    const TileCost& c = f32 ? kCost32[t] : kCost[t];
    const int64_t bm = f32 ? kTileM32[t] : kTileM[t], bn = (f32 ? kTileN32[t] : kTileN[t]) / halves;
    const double tiles = (double)((rows + bm - 1) / bm) * (double)((cols + bn - 1) / bn);
    for (int s : kSplits) {
      if (s > 1 && (2 * s > stages || tiles * s > 8.0 * cus)) break;
      const double per = std::ceil(stages / s), blocks = std::ceil(tiles * s / cus);
      const double rounds = std::ceil(blocks / c.resident);
      double us = std::max(blocks * c.stage, rounds * c.alone) * per + rounds * c.ends;
      if (s > 1) us += f32 ? 2.1 + 0.2 * part_mb * s : 5.0 + 0.114 * part_mb * s;
      if (us < least) least = us, best = {t, s};
    }
  }
  return best;
}

hipError_t launch_product_bf16(Form form, const ProductPlan& plan, ProductArgs a, hipStream_t stream) {
  return mm::launch<false>(form, plan, a, stream);
}

}  // namespace pointid
