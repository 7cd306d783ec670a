// The matrix-core products of fp32 operands: every value is the sum of three bf16 values
// (its rounding, the remainder's rounding, and the rest: 8 + 8 + 8 bits), and a product is
// the 6 products of parts whose orders add up to less than 3, the smallest first; what is
// left out is at most 2^-24 of a product, its root mean square 2^-27.  bf16 ends at 2^-133, so
// that a value below 2^-110 is off by up to 2^-134.
//
// Values are read as fp32, 32 inner indices at a time, while the stage before multiplies,
// cut in registers and written to shared memory as three planes laid out as in the 16-bit
// kernels (layers_mm.h); two stages.  A stage's 6 products share its fragments, so they
// read half of what 6 passes over 16-bit planes would, and no pass lays planes out first.
//
// Bound by power where there is work for all CUs (4096^3: 593-597 us, 231 TFLOP/s, which is
// 1.38 PFLOP/s of bf16 products); below that by a stage's chain of loading, cutting and
// multiplying, 1 to 2 us, with one 128 x 128 or 256 x 128 tile a CU (235 x 2304 x (2 x 1021):
// 25 us and 6 of the join; 50 % MFMA busy in a gradient's pair of products of 1693 x 1024 x
// (2 x 2048)).  Reading a stage's first fragments during the last products of the one before
// (as the 16-bit kernels do), and loads two stages ahead, gained nothing.
#include "layers_mm.h"

namespace pointid {
namespace mm {
namespace {

constexpr int kBK32 = 32;                   // inner indices of a stage

// One operand's tile: kInner: [kSide][32], else [32][kSide].  A thread reads 4 values at a
// time along the rows.
template <bool kInner, int kSide, int kThreads>
struct Tile32 {
  static constexpr int kPieces = kInner ? kBK32 / 4 : kSide / 4;     // of 4 values, of a row
  static constexpr int kRows = kInner ? kSide : kBK32;
  static constexpr int kPlane = kSide * kBK32 * 2;
  static constexpr int kLoads = kRows * kPieces / kThreads;
  static_assert(kLoads * kThreads == kRows * kPieces, "whole loads");

  uint32_t offset[kLoads];                  // of the thread's values from the tile's origin
  uint16_t to[kLoads];                      // where their parts go in a plane
  int16_t inner[kLoads];                    // the first's inner index
  int16_t count[kLoads];                    // kInner: 4, or 0 past the rows; else columns that exist

  __device__ __forceinline__ void init(int tid, int64_t side0, int64_t sides, int64_t ld) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = i * kThreads + tid, row = at / kPieces, piece = at % kPieces;
      const int64_t side = side0 + (kInner ? row : piece * 4);
      inner[i] = (int16_t)(kInner ? piece * 4 : row);
      offset[i] = (uint32_t)((row * ld + piece * 4) * 4);
      const int64_t n = sides - side;
      count[i] = (int16_t)(n <= 0 ? 0 : kInner || n > 4 ? 4 : n);
      const int pitch = kInner ? kBK32 * 2 : kSide * 2;
      to[i] = (uint16_t)(row * pitch + place<kInner, kInner ? kBK32 / 8 : kSide / 8>(row, piece / 2) * 16 + piece % 2 * 8);
    }
  }
  // whole: every group of 4 values exists as a whole or not at all
  __device__ __forceinline__ void load(const char* origin, int left, bool whole, float4 (&v)[kLoads]) const {
    const __amdgpu_buffer_rsrc_t r =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(origin), (short)0, (int)kNowhere, 0x00020000);
    if (whole) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        v[i] = __builtin_bit_cast(
            float4, __builtin_amdgcn_raw_buffer_load_b128(r, count[i] && inner[i] < left ? offset[i] : kNowhere, 0, 0));
      return;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool there = kInner ? count[i] && inner[i] + j < left : j < count[i] && inner[i] < left;
        f[j] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, there ? offset[i] + 4 * j : kNowhere, 0, 0));
      }
      v[i] = make_float4(f[0], f[1], f[2], f[3]);
    }
  }
  // The three parts of two values.  kCare: an infinity or NaN stands in the last part (which
  // multiplies the first part of the other operand alone) behind a 1 of its sign and a 0, and
  // so goes through as in fp32, and the first part of the largest values, which would round to
  // an infinity, is the largest bf16.
  template <bool kCare>
  static __device__ __forceinline__ void cut(float a, float b, uint32_t (&part)[3]) {
    auto rest = [&](uint32_t h) {
      a -= __uint_as_float(h << 16);
      b -= __uint_as_float(h & 0xFFFF0000u);
      return h;
    };
    if constexpr (kCare) {
      constexpr float kMost = 3.38953139e38f;
      const bool fa = __builtin_isfinite(a), fb = __builtin_isfinite(b);
      const float most_a = fa ? kMost : 1.f, most_b = fb ? kMost : 1.f;
      part[0] = rest(Op16<false>::pack(__builtin_amdgcn_fmed3f(a, -most_a, most_a), __builtin_amdgcn_fmed3f(b, -most_b, most_b)));
      part[1] = rest(Op16<false>::pack(fa ? a : 0.f, fb ? b : 0.f));
    } else {
      part[0] = rest(Op16<false>::pack(a, b));
      part[1] = rest(Op16<false>::pack(a, b));
    }
    part[2] = Op16<false>::pack(a, b);
  }
  // The parts of the values to the three planes at `tile`, kPitch bytes apart.
  template <bool kCare, int kPitch>
  __device__ __forceinline__ void store(char* tile, const float4 (&v)[kLoads]) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      uint32_t x[3], y[3];
      cut<kCare>(v[i].x, v[i].y, x);
      cut<kCare>(v[i].z, v[i].w, y);
#pragma unroll
      for (int p = 0; p < 3; ++p) *reinterpret_cast<uint2*>(tile + p * kPitch + to[i]) = make_uint2(x[p], y[p]);
    }
  }
};

// Shared memory of a block: two stages of three planes; the end fits where they were.
template <int kBM, int kBN, int kWM, int kWN>
constexpr int shared_bytes32() {
  constexpr int kStages = 2 * 3 * (kBM + kBN) * kBK32 * 2;
  static_assert(kWM * kWN * kEndWave <= kStages, "the end's part");
  return kStages;
}

template <int kForm, int kHalves, int kBM, int kBN, int kWM, int kWN>
__device__ __forceinline__ void product_f32_block(const ProductArgs& a, uint32_t block, char* smem) {
  constexpr int kThreads = 64 * kWM * kWN;
  constexpr bool kLeftInner = kForm != kDw, kRightInner = kForm == kDx;
  static_assert(!kRightInner || kHalves == 1, "dx has one half");
  constexpr int kHN = kBN / 2;
  constexpr int kFragsM = kBM / kWM / 16, kFragsN = 4;
  static_assert(kBN / kWN == 64, "a wave takes 64 columns");
  using Left = Tile32<kLeftInner, kBM, kThreads>;
  using Right = Tile32<kRightInner, kHN, kThreads>;
  // a stage: the left operand's planes, then the right one's, half after half in each
  constexpr int kLeftBytes = 3 * Left::kPlane, kStage = kLeftBytes + 6 * Right::kPlane;

  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int wm = wave / kWN, wn = wave % kWN;
  const Place at = block_place(a, block);
  const int64_t row0 = at.tm * kBM;
  const int64_t col0 = at.tn * (kHalves == 2 ? kHN : kBN), col1 = kHalves == 2 ? col0 : col0 + kHN;
  Left left;
  Right right0, right1;
  left.init(tid, row0, a.end.rows, a.ld_left);
  right0.init(tid, col0, a.end.cols, a.ld_right);
  right1.init(tid, col1, a.end.cols, a.ld_right);
  Frags<kLeftInner, kBM, kFragsM, kBK32> lf;
  Frags<kRightInner, kHN, kFragsN, kBK32> rf;
  lf.init(lane, [&](int i, int* tile) {
    *tile = 0;
    return wm * (kBM / kWM) + 16 * i;
  });
  rf.init(lane, [&](int i, int* tile) {
    const int col = kHalves == 2 ? i / 2 * kHN + wn * 32 + i % 2 * 16 : wn * 64 + 16 * i;
    *tile = kLeftBytes + col / kHN * Right::kPlane;
    return col % kHN;
  });

  const int stages = a.split_each + (at.split < (uint32_t)a.split_more);
  const uint32_t first = at.split * a.split_each + (at.split < (uint32_t)a.split_more ? at.split : a.split_more);
  const int term0 = (int)(first / (uint32_t)a.stages);
  int to_load, term, k0;
  const int64_t left_step = (kLeftInner ? kBK32 : kBK32 * a.ld_left) * 4;
  const int64_t right_step = (kRightInner ? kBK32 : kBK32 * a.ld_right) * 4;
  const bool whole_left = kLeftInner ? a.inner % 4 == 0 : a.end.rows % 4 == 0;
  const bool whole_right = kRightInner ? a.inner % 4 == 0 : a.end.cols % 4 == 0;

  float4 lv[Left::kLoads], rv0[Right::kLoads], rv1[Right::kLoads];
  auto load = [&] {
    const Term& t = a.term[term];
    const int64_t s = k0 / kBK32;
    const int left_of = a.inner - k0;
    left.load(static_cast<const char*>(t.left) + (kLeftInner ? row0 * a.ld_left : row0) * 4 + s * left_step, left_of,
              whole_left, lv);
    right0.load(static_cast<const char*>(t.right0) + (kRightInner ? col0 * a.ld_right : col0) * 4 + s * right_step,
                left_of, whole_right, rv0);
    right1.load(static_cast<const char*>(kHalves == 2 ? t.right1 : t.right0) +
                    (kRightInner ? col1 * a.ld_right : col1) * 4 + s * right_step,
                left_of, whole_right, rv1);
    k0 += kBK32;
    if (k0 >= a.inner) k0 = 0, ++term;
    --to_load;
  };
  floatx4 acc[kFragsM][kFragsN];
  uint4 r[3][kFragsN], l[2][3];
  auto read_left = [&](const char* tile, int i) {
#pragma unroll
    for (int p = 0; p < 3; ++p) l[i % 2][p] = lf.read(tile + p * Left::kPlane, i, 0);
  };
  auto multiply = [&](int i) {
#pragma unroll
    for (int order = 2; order >= 0; --order)
#pragma unroll
      for (int p = order; p >= 0; --p)
#pragma unroll
        for (int j = 0; j < kFragsN; ++j) acc[i][j] = mfma<false>(r[order - p][j], l[i % 2][p], acc[i][j]);
  };
  // Of the two waves that share a SIMD one cuts and stores the next stage before it multiplies,
  // the other halfway, so that one cuts while the other multiplies (both halfway: 2048 x 4096 x
  // 2048 176 us for 173, its dx 172 for 164; the second at the end: 177).
  const bool early = kWM * kWN == 8 && wave < 4;
  auto sum = [&](auto care) {
    auto store = [&](int stage) {
      char* tile = smem + stage * kStage;
      left.template store<care, Left::kPlane>(tile, lv);
      right0.template store<care, 2 * Right::kPlane>(tile + kLeftBytes, rv0);
      right1.template store<care, 2 * Right::kPlane>(tile + kLeftBytes + Right::kPlane, rv1);
    };
    to_load = stages;
    term = term0;
    k0 = (int)(first - (uint32_t)term0 * a.stages) * kBK32;
#pragma unroll
    for (int i = 0; i < kFragsM; ++i)
#pragma unroll
      for (int j = 0; j < kFragsN; ++j) acc[i][j] = floatx4{};
    if (stages == 0) return;
    load();
    store(0);
    if (to_load > 0) load();
    __syncthreads();
    for (int it = 0; it < stages; ++it) {
      const int stage = it % 2;
      const char* tile = smem + stage * kStage;
#pragma unroll
      for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int j = 0; j < kFragsN; ++j) r[p][j] = rf.read(tile + p * 2 * Right::kPlane, j, 0);
      read_left(tile, 0);
      auto next = [&] {
        if (it + 1 == stages) return;
        store(stage ^ 1);
        if (to_load > 0) load();
      };
      if (early) next();
#pragma unroll
      for (int i = 0; i < kFragsM; ++i) {
        if (i + 1 < kFragsM) read_left(tile, i + 1);
        multiply(i);
        if (i == (kFragsM - 1) / 2 && !early) next();
      }
      __syncthreads();
    }
  };
  sum(std::false_type{});
  // A value whose first part is not finite makes all sums of its row or column so: these are
  // made again with care (whole blocks, so that the loop does not pay for it: with the clamp
  // in it 4096^3 took 607 us for 593).
  float all = 0.f;
#pragma unroll
  for (int i = 0; i < kFragsM; ++i)
#pragma unroll
    for (int j = 0; j < kFragsN; ++j)
#pragma unroll
      for (int c = 0; c < 4; ++c) all = __builtin_fmaf(acc[i][j][c], 0.f, all);
  if (__syncthreads_or(all != 0.f)) sum(std::true_type{});
  end_tile<POINTID_FP32, kHalves, kFragsM>(a.end, acc, reinterpret_cast<float*>(smem) + wave * kEndWave / 4,
                                                    lane, at.split, row0 + wm * (kBM / kWM),
                                                    col0 + wn * (kHalves == 2 ? 32 : 64), 1.f);
}

template <int kForm, int kHalves, int kBM, int kBN, int kWM, int kWN>
__global__ void __launch_bounds__(64 * kWM * kWN) product_f32_kernel(ProductArgs a) {
  __shared__ __align__(1024) char smem[shared_bytes32<kBM, kBN, kWM, kWN>()];
  product_f32_block<kForm, kHalves, kBM, kBN, kWM, kWN>(a, blockIdx.x, smem);
}
template <int kHalves, int kBM, int kBN, int kWM, int kWN>
__global__ void __launch_bounds__(64 * kWM * kWN) pair_f32_kernel(PairArgs a) {
  __shared__ __align__(1024) char smem[shared_bytes32<kBM, kBN, kWM, kWN>()];
  pair_block<64 * kWM * kWN>(
      a, smem, [&](const ProductArgs& p, uint32_t block) { product_f32_block<kDx, 1, kBM, kBN, kWM, kWN>(p, block, smem); },
      [&](const ProductArgs& p, uint32_t block) { product_f32_block<kDw, kHalves, kBM, kBN, kWM, kWN>(p, block, smem); });
}

template <int kForm, int kHalves>
hipError_t launch_tile32(int tile, ProductArgs& a, hipStream_t stream) {
  const int bm = kTileM32[tile], bn = kTileN32[tile] / (kHalves == 2 ? 2 : 1);
  const int64_t blocks = spread(a, bm, bn, kBK32);
  if (blocks < 1 || a.end.dtype != POINTID_FP32) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  switch (tile) {
    case 0: return launch_kernel(product_f32_kernel<kForm, kHalves, 256, 128, 4, 2>, grid, dim3(512), 0, stream, a);
    case 1: return launch_kernel(product_f32_kernel<kForm, kHalves, 128, 128, 4, 2>, grid, dim3(512), 0, stream, a);
    case 2: return launch_kernel(product_f32_kernel<kForm, kHalves, 64, 128, 2, 2>, grid, dim3(256), 0, stream, a);
    case 3: return launch_kernel(product_f32_kernel<kForm, kHalves, 64, 64, 4, 1>, grid, dim3(256), 0, stream, a);
  }
  return hipErrorInvalidValue;
}

template <int kHalves>
hipError_t launch_pair_tile32(int tile, PairArgs& a, hipStream_t stream) {
  const int64_t blocks = spread_pair(a, kTileM32[tile], kTileN32[tile], kBK32);
  if (blocks < 1 || a.dx.end.dtype != POINTID_FP32 || a.dw.end.dtype != POINTID_FP32) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  switch (tile) {
    case 0: return launch_kernel(pair_f32_kernel<kHalves, 256, 128, 4, 2>, grid, dim3(512), 0, stream, a);
    case 1: return launch_kernel(pair_f32_kernel<kHalves, 128, 128, 4, 2>, grid, dim3(512), 0, stream, a);
    case 2: return launch_kernel(pair_f32_kernel<kHalves, 64, 128, 2, 2>, grid, dim3(256), 0, stream, a);
    case 3: return launch_kernel(pair_f32_kernel<kHalves, 64, 64, 4, 1>, grid, dim3(256), 0, stream, a);
  }
  return hipErrorInvalidValue;
}

}  // namespace
}  // namespace mm

hipError_t launch_product_f32(Form form, const ProductPlan& plan, ProductArgs a, hipStream_t stream) {
  a.splits = plan.splits;
  const bool two = a.end.halves == 2;
  switch (form) {
    case kForward:
      return two ? mm::launch_tile32<kForward, 2>(plan.tile, a, stream) : mm::launch_tile32<kForward, 1>(plan.tile, a, stream);
    case kDx: return two ? hipErrorInvalidValue : mm::launch_tile32<kDx, 1>(plan.tile, a, stream);
    case kDw: return two ? mm::launch_tile32<kDw, 2>(plan.tile, a, stream) : mm::launch_tile32<kDw, 1>(plan.tile, a, stream);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_pair_f32(int tile, const ProductArgs& dx, const ProductArgs& dw, const SumsJobs& sums, hipStream_t stream) {
  mm::PairArgs a;
  a.dx = dx, a.dw = dw, a.sums = sums;
  return dw.end.halves == 2 ? mm::launch_pair_tile32<2>(tile, a, stream) : mm::launch_pair_tile32<1>(tile, a, stream);
}

}  // namespace pointid
