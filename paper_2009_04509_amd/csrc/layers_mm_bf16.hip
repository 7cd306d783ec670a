// The matrix-core products of bf16 operands, and the choice of tiles and splits of all types.
#include "layers_mm.h"

#include <algorithm>
#include <cmath>

namespace pointid {

namespace {

// us of a tile shape, fitted to sweeps of tiles and splits over 32 products of all forms
// from 4 x 12288 x 4096 to 16384 x 4096 x 1024 (70 in fp32): a stage of 64 inner indices when
// `resident` blocks share a CU (each) and of a block alone, and a block's start and end.
// The choice by them takes half a percent more than the fastest measured on average, at
// worst 6 % (fp32 15).
struct TileCost {
  double stage, alone, ends;
  int resident;
};
constexpr TileCost kCost[kTiles] = {
    {1.25, 1.25, 8.5, 1}, {0.555, 0.555, 2.6, 1}, {0.515, 0.617, 2.6, 2}, {0.314, 0.463, 1.7, 3}};
constexpr TileCost kCost32[kTiles32] = {{4.53, 4.53, 3.0, 1}, {2.76, 2.76, 2.4, 1}, {1.58, 2.79, 0.8, 2}, {1.0, 1.8, 0.7, 3}};

constexpr int kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128};

struct Timed {
  ProductPlan plan;
  double us;
};

// A product's tiles of shape t, the stages of each, and the MB of fp32 results that a split
// of its sum writes and reads.
struct Sizes {
  double tiles, stages, part_mb;
};
Sizes sizes_of(bool f32, int t, int64_t rows, int64_t cols, int halves, int64_t inner, int terms) {
  const int64_t bm = f32 ? kTileM32[t] : kTileM[t], bn = (f32 ? kTileN32[t] : kTileN[t]) / halves;
  return {(double)((rows + bm - 1) / bm) * (double)((cols + bn - 1) / bn), (double)((inner + 63) / 64) * terms,
          8e-6 * (double)rows * (double)cols * halves};
}
// Whether a sum may be split so: two stages each, and not many more blocks than the card holds.
bool may_split(const Sizes& z, int splits, int cus) {
  return splits == 1 || (2 * splits <= z.stages && z.tiles * splits <= 8.0 * cus);
}
double join_cost(bool f32, const Sizes& z, int splits) {
  return splits == 1 ? 0 : f32 ? 6.0 + 0.138 * z.part_mb * splits : 1.4 + 0.16 * z.part_mb * splits;
}

Timed least_cost(bool f32, int64_t rows, int64_t cols, int halves, int64_t inner, int terms, int cus) {
  Timed best = {{0, 1}, 1e300};
  for (int t = 0; t < (f32 ? kTiles32 : kTiles); ++t) {
    const TileCost& c = f32 ? kCost32[t] : kCost[t];
    const Sizes z = sizes_of(f32, t, rows, cols, halves, inner, terms);
    for (int s : kSplits) {
      if (!may_split(z, s, cus)) break;
      const double per = std::ceil(z.stages / s), blocks = std::ceil(z.tiles * s / cus);
      const double rounds = std::ceil(blocks / c.resident);
      const double us = std::max(blocks * c.stage, rounds * c.alone) * per + rounds * c.ends + join_cost(f32, z, s);
      if (us < best.us) best = {{t, s}, us};
    }
  }
  return best;
}

}  // namespace

// The tile and split that the costs above put first.  Large tiles read their operands fewer
// times (bf16 4096 x 1024 x 4096: 37 us in 256 x 256 tiles, 41 in 128 x 128, 49 in 64 x 128);
// small ones fill the CUs where there are few (2048^3: 26 in 64 x 128, 44 in split 256 x 256;
// its gated form 37 in 128 x 128, 49 and 51 in the others); three stages hide the loads of
// one 128 x 128 tile a CU (4096 x 4096 x 1024: 43 against 50), two leave room for a second.
// fp32: 2048^3 96 in 128 x 128 tiles, 136 in 64 x 64; 308 x 7121 x 944 47 in 64 x 128, 53 in
// 64 x 64, 57 in 128 x 128; 235 x 128 x 32 8.7 in 64 x 64, 10.4 in 64 x 128 (the chain of a
// stage is shorter); a gated 3257 x 2532 x 285 82 in 256 x 128, 89 in 64 x 128.
ProductPlan plan_product(bool f32, int64_t rows, int64_t cols, int halves, int64_t inner, int terms, int cus) {
  return least_cost(f32, rows, cols, halves, inner, terms, cus).plan;
}

// Together, the blocks of one product fill the CUs that the other leaves, and no second
// launch waits for the first's last blocks (bf16, dx and dW of 1693 x 1024 x 2048: 23 us
// against 42 by two launches; of 4096 x 1024 x 4096: 72 against 84; fp32 2048^3: 170 against
// 201), and what one writes goes along with what the other reads (1693 x 92928 x 128: 198
// against 220).  16-bit tiles of 256 x 256
// are better alone (16384 x 1024 x 1024: 86 against 90; 4096^3: 214 against 270 in smaller ones).
// A CU's time is that of its share of the stages, or of the longest block's: as many stages as
// the other's blocks have beside them, the rest alone.  Two launches cost 6 us more than their
// blocks, a second join 3.4 (fitted to 35 shapes; within 5 % of the fastest).
PairPlan plan_pair(bool f32, int64_t m, int64_t k, int64_t n, int halves, int parts, int cus) {
  PairPlan best = {-1, 1, 1};
  double least = least_cost(f32, m, k, 1, n, halves * parts, cus).us +
                 least_cost(f32, k, n, halves, m, parts, cus).us + 6.0;
  for (int t = f32 ? 0 : 1; t < (f32 ? kTiles32 : kTiles); ++t) {
    const TileCost& c = f32 ? kCost32[t] : kCost[t];
    const Sizes dx = sizes_of(f32, t, m, k, 1, n, halves * parts), dw = sizes_of(f32, t, k, n, halves, m, parts);
    for (int s : kSplits) {
      if (!may_split(dx, s, cus)) break;
      for (int r : kSplits) {
        if (!may_split(dw, r, cus)) break;
        const double x = std::ceil(dx.stages / s), w = std::ceil(dw.stages / r), count = dx.tiles * s + dw.tiles * r;
        const double blocks = std::ceil(count / cus), beside = std::min(blocks, (double)c.resident);
        const double work = (dx.tiles * s * x + dw.tiles * r * w) / count * blocks * c.stage;
        const double longest = blocks > 1 ? std::min(x, w) * std::max(beside * c.stage, c.alone) + std::abs(x - w) * c.alone
                                          : std::max(x, w) * c.alone;
        const double us = std::max(work, longest) + std::ceil(blocks / c.resident) * c.ends + join_cost(f32, dx, s) +
                          join_cost(f32, dw, r) + 2.0 * (s > 1) + 2.0 * (r > 1);
        if (us < least) least = us, best = {t, s, r};
      }
    }
  }
  return best;
}

hipError_t launch_product_bf16(Form form, const ProductPlan& plan, ProductArgs a, hipStream_t stream) {
  return mm::launch<false>(form, plan, a, stream);
}

hipError_t launch_pair_bf16(int tile, const ProductArgs& dx, const ProductArgs& dw, const SumsJobs& sums, hipStream_t stream) {
  return mm::launch_pair<false>(tile, dx, dw, sums, stream);
}

}  // namespace pointid
