// The matrix-core products of bf16 operands, and the choice of tiles and splits of all types.
#include "layers_mm.h"

#include <algorithm>
#include <cmath>

namespace pointid {

namespace {

// us of a tile shape, fitted to sweeps of tiles and splits over 32 products of all forms
// from 4 x 12288 x 4096 to 16384 x 4096 x 1024 (24 in fp32): a stage of 64 inner indices when
// `resident` blocks share a CU (each) and of a block alone, and a block's start and end.
// The choice by them is the fastest measured or within 6 % of it, half a percent on average.
struct TileCost {
  double stage, alone, ends;
  int resident;
};
constexpr TileCost kCost[kTiles] = {
    {1.25, 1.25, 8.5, 1}, {0.555, 0.555, 2.6, 1}, {0.515, 0.617, 2.6, 2}, {0.314, 0.463, 1.7, 3}};
constexpr TileCost kCost32[kTiles32] = {{4.53, 4.53, 3.0, 1}, {2.76, 2.76, 2.4, 1}, {1.58, 2.79, 0.8, 2}};

}  // namespace

// The tile and split that the costs above put first.  Large tiles read their operands fewer
// times (bf16 4096 x 1024 x 4096: 37 us in 256 x 256 tiles, 41 in 128 x 128, 49 in 64 x 128);
// small ones fill the CUs where there are few (2048^3: 26 in 64 x 128, 44 in split 256 x 256;
// its gated form 37 in 128 x 128, 49 and 51 in the others); three stages hide the loads of
// one 128 x 128 tile a CU (4096 x 4096 x 1024: 43 against 50), two leave room for a second.
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
      if (s > 1) us += f32 ? 6.0 + 0.138 * part_mb * s : 1.4 + 0.16 * part_mb * s;
      if (us < least) least = us, best = {t, s};
    }
  }
  return best;
}

hipError_t launch_product_bf16(Form form, const ProductPlan& plan, ProductArgs a, hipStream_t stream) {
  return mm::launch<false>(form, plan, a, stream);
}

}  // namespace pointid
