// Products on the matrix cores (16-bit operands, fp32 sums), one template for the three
// forms of layers.h.
//
// A block computes kBM x kBN results with 32x32x16 MFMAs.  Both operands go through
// shared memory, 64 inner indices at a time, two stages, written by loads that go there
// directly (16 bytes a lane).  An operand whose rows run along the inner index (x and dz
// of dx and forward's x) is read as fragments with 16-byte reads; one whose rows are
// indexed by the inner index (W of the forward form, both of dW) with the transposing
// read, 4 x 16 values at a time, so no form needs a transposed copy of anything.
//
// The results come out with the right operand as the MFMA's first, so a lane holds one
// row's columns: after a swap of halves 16 consecutive ones, and a lane and the one 32
// away a whole block of 32 for the 8-bit checkpoint.
//
// Pieces of 16 bytes stand in shared memory in a permuted order that the loads apply to
// their global addresses.  Rows of 64 inner indices (128 bytes): piece p of row r at
// p ^ (r / 2 % 8), so that 16 lanes reading one piece of 16 rows touch all banks.  Rows of
// columns: the 64-byte group g of row r at g ^ (r % 4) (rows of 128 bytes: g ^ (r / 2 % 2)),
// so that the 4 rows of a transposing read do.
#pragma once

#include "internal.h"
#include "layers_end.h"

namespace pointid {
namespace mm {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

constexpr int kBK = 64;                     // inner indices of a stage
constexpr uint32_t kNowhere = 0x80000000u;  // an offset past the resource's range: reads 0

// The piece's place in a row of kPieces pieces of 16 bytes; kInner: rows along the inner index.
template <bool kInner, int kPieces>
__device__ __forceinline__ int place(int row, int piece) {
  if constexpr (kInner) return piece ^ ((row >> 1) & 7);
  if constexpr (kPieces >= 16) return piece ^ ((row & 3) << 2);
  return piece ^ (((row >> 1) & 1) << 2);
}

__device__ __forceinline__ intx4 resource(const void* base) {
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  intx4 r;
  r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)b);
  r[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32) & 0xFFFF);
  r[2] = (int)kNowhere;
  r[3] = 0x00020000;
  return r;
}

// 64 lanes x 16 bytes straight to shared memory at `lds` (the wave's), lane after lane.
// Nothing is returned; the stage's wait covers it.
__device__ __forceinline__ void load_to_lds(intx4 rsrc, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(lds), "v"(offset), "s"(rsrc) : "memory");
}

// One operand's tile of kSide rows or columns: kInner: [kSide][64], else [64][kSide].
template <bool kInner, int kSide, int kThreads>
struct Tile {
  static constexpr int kPieces = kInner ? kBK / 8 : kSide / 8;       // of a row
  static constexpr int kRows = kInner ? kSide : kBK;
  static constexpr int kBytes = kSide * kBK * 2;
  static constexpr int kLoads = kRows * kPieces / kThreads;
  static_assert(kLoads * kThreads == kRows * kPieces, "whole loads");

  uint32_t offset[kLoads];                  // of the lane's pieces from the tile's origin
  int16_t inner[kLoads];                    // first inner index of the piece

  // side0: the tile's first row or column of `sides`
  __device__ __forceinline__ void init(int tid, int64_t side0, int64_t sides, int64_t ld) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = i * kThreads + tid, row = at / kPieces;
      const int piece = place<kInner, kPieces>(row, at % kPieces);       // its own inverse
      const int side = kInner ? row : piece * 8;
      inner[i] = (int16_t)(kInner ? piece * 8 : row);
      offset[i] = side0 + side < sides ? (uint32_t)((row * ld + piece * 8) * 2) : kNowhere;
    }
  }
  // The stage from inner index k0 of `inners` on; `origin` points at (side0, 0).
  __device__ __forceinline__ void load(const char* origin, int64_t k0, int64_t inners, int64_t ld, uint32_t lds,
                                       int wave) const {
    const intx4 r = resource(origin + (kInner ? k0 : k0 * ld) * 2);
    const int left = inners - k0 < kBK ? (int)(inners - k0) : kBK;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      load_to_lds(r, inner[i] < left ? offset[i] : kNowhere, lds + (i * kThreads + wave * 64) * 16);
  }
};

// Fragments: 8 consecutive inner indices of one row or column a lane (lane % 32; lanes of
// 32 and more the next 8), for kFrags groups of 32 rows or columns from side0 on.
template <bool kInner, int kSide, int kFrags>
struct Frags {
  int base[kInner ? 4 : kFrags];
  __device__ __forceinline__ void init(int lane, int side0) {
    if constexpr (kInner) {
      const int row = side0 + lane % 32;
#pragma unroll
      for (int s = 0; s < 4; ++s) base[s] = row * 128 + place<true, 8>(row, 2 * s + lane / 32) * 16;
    } else {
      // the lane's address in a read of 4 rows x 16 columns by 16 lanes
      const int row = lane / 32 * 8 + lane % 16 / 4;
#pragma unroll
      for (int i = 0; i < kFrags; ++i) {
        const int col = side0 + 32 * i + lane / 16 % 2 * 16 + lane % 4 * 4;
        base[i] = row * (kSide * 2) + place<false, kSide / 8>(row, col / 8) * 16 + col % 8 * 2;
      }
    }
  }
  // inner indices 16 s .. 16 s + 15 of group i
  __device__ __forceinline__ uint4 read(const char* tile, int i, int s) const {
    if constexpr (kInner) {
      return *reinterpret_cast<const uint4*>(tile + base[s] + i * 32 * 128);
    } else {
      typedef __attribute__((address_space(3))) shortx4 LdsShort4;
      const char* p = tile + base[i] + s * 16 * kSide * 2;
      const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4*)p);
      const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4*)(p + 4 * kSide * 2));
      const uint2 l = __builtin_bit_cast(uint2, lo), h = __builtin_bit_cast(uint2, hi);
      return make_uint4(l.x, l.y, h.x, h.y);
    }
  }
};

template <bool kFp16>
__device__ __forceinline__ floatx16 mfma(const uint4& a, const uint4& b, const floatx16& c) {
  if constexpr (kFp16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a), __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// A lane's 16 sums of a 32 x 32 result (columns 8 j + 4 (lane / 32) + t of row lane % 32) ->
// columns 16 (lane / 32) .. + 15 of that row.
__device__ __forceinline__ void consecutive(const floatx16& c, float* v) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(c[4 * j + t]), __float_as_uint(c[4 * j + 8 + t]),
                                                      false, false);
      v[8 * j + t] = __uint_as_float(q[0]);
      v[8 * j + 4 + t] = __uint_as_float(q[1]);
    }
}

// All loads to shared memory of this wave done, then the block's barrier.
__device__ __forceinline__ void stage_ready() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <bool kFp16, int kForm, int kHalves, int kBM, int kBN, int kWM, int kWN>
__global__ void __launch_bounds__(64 * kWM * kWN) product_kernel(ProductArgs a) {
  constexpr int kThreads = 64 * kWM * kWN;
  constexpr bool kLeftInner = kForm != kDw, kRightInner = kForm == kDx;
  constexpr int kHN = kBN / 2;                           // columns of each half of the tile
  constexpr int kFragsM = kBM / kWM / 32;
  static_assert(kHN / kWN == 32, "a wave takes 32 columns of each half");
  using Left = Tile<kLeftInner, kBM, kThreads>;
  using Right = Tile<kRightInner, kHN, kThreads>;
  constexpr int kStage = Left::kBytes + 2 * Right::kBytes;
  __shared__ __align__(1024) char smem[2 * kStage];

  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int wm = wave / kWN, wn = wave % kWN;

  // Blocks go to the 8 XCDs in turn: each XCD takes a contiguous stretch of the tiles, in
  // groups of 8 rows of tiles walked column by column, so that the blocks which run
  // together on an XCD share operands in its L2.
  const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
  const int64_t all = tiles * a.splits;
  const int64_t each = all / 8, more = all % 8, xcd = blockIdx.x % 8;
  int64_t id = xcd * each + (xcd < more ? xcd : more) + blockIdx.x / 8;
  const int split = (int)(id / tiles);
  id -= split * tiles;
  constexpr int kGroup = 8;
  const int64_t group = id / ((int64_t)kGroup * a.tiles_n), in = id - group * kGroup * a.tiles_n;
  const int64_t rows_here = a.tiles_m - group * kGroup < kGroup ? a.tiles_m - group * kGroup : kGroup;
  const int64_t tm = group * kGroup + in % rows_here, tn = in / rows_here;

  const int64_t row0 = tm * kBM;
  const int64_t col0 = tn * (kHalves == 2 ? kHN : kBN), col1 = kHalves == 2 ? col0 : col0 + kHN;
  Left left;
  Right right0, right1;
  left.init(tid, row0, a.end.rows, a.ld_left);
  right0.init(tid, col0, a.end.cols, a.ld_right);
  right1.init(tid, col1, a.end.cols, a.ld_right);
  Frags<kLeftInner, kBM, kFragsM> lf;
  Frags<kRightInner, kHN, 1> rf;
  lf.init(lane, wm * (kBM / kWM));
  rf.init(lane, wn * 32);

  const int64_t its = (a.inner + kBK - 1) / kBK, total = its * a.terms;
  int64_t it = total * split / a.splits;
  const int64_t end = total * (split + 1) / a.splits;
  int term = (int)(it / its);
  int64_t k0 = (it - term * its) * kBK;
  const int64_t left_at = (kLeftInner ? row0 * a.ld_left : row0) * 2;
  const int64_t right_at0 = (kRightInner ? col0 * a.ld_right : col0) * 2;
  const int64_t right_at1 = (kRightInner ? col1 * a.ld_right : col1) * 2;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;

  auto issue = [&](int stage) {
    const uint32_t at = lds0 + stage * kStage;
    const Term& t = a.term[term];
    left.load(static_cast<const char*>(t.left) + left_at, k0, a.inner, a.ld_left, at, wave);
    right0.load(static_cast<const char*>(t.right0) + right_at0, k0, a.inner, a.ld_right, at + Left::kBytes, wave);
    right1.load(static_cast<const char*>(kHalves == 2 ? t.right1 : t.right0) + right_at1, k0, a.inner, a.ld_right,
                at + Left::kBytes + Right::kBytes, wave);
    k0 += kBK;
    if (k0 >= a.inner) k0 = 0, ++term;
  };

  floatx16 acc[kFragsM][2] = {};
  auto compute = [&](int stage) {
    const char* tl = smem + stage * kStage;
    const char* t0 = tl + Left::kBytes;
    const char* t1 = t0 + Right::kBytes;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const uint4 r0 = rf.read(t0, 0, s), r1 = rf.read(t1, 0, s);
#pragma unroll
      for (int i = 0; i < kFragsM; ++i) {
        const uint4 l = lf.read(tl, i, s);
        acc[i][0] = mfma<kFp16>(r0, l, acc[i][0]);
        acc[i][1] = mfma<kFp16>(r1, l, acc[i][1]);
      }
    }
  };

  int stage = 0;
  if (it < end) {
    issue(0);
    stage_ready();
    for (; it + 1 < end; ++it) {
      issue(stage ^ 1);
      compute(stage);
      stage_ready();
      stage ^= 1;
    }
    compute(stage);
  }

  // One copy of the end's code: the sums of each turn are moved to where it takes them from.
  constexpr int kTurns = kHalves == 2 ? kFragsM : 2 * kFragsM;
#pragma nounroll
  for (int turn = 0; turn < kTurns; ++turn) {
    floatx16 c0 = {}, c1 = {};
    static_for<kTurns>([&](auto t) {
      if (turn == t) {
        c0 = acc[kHalves == 2 ? t : t / 2][kHalves == 2 ? 0 : t % 2];
        if constexpr (kHalves == 2) c1 = acc[t][1];
      }
    });
    const int64_t row = row0 + wm * (kBM / kWM) + 32 * (kHalves == 2 ? turn : turn / 2) + lane % 32;
    const int64_t col = (kHalves == 2 || turn % 2 == 0 ? col0 : col1) + wn * 32 + lane / 32 * 16;
    const bool live = row < a.end.rows;
    float v[kHalves][16];
    consecutive(c0, v[0]);
    if constexpr (kHalves == 2) consecutive(c1, v[1]);
    if (a.end.mode == kEndPartial) {
#pragma unroll
      for (int h = 0; h < kHalves; ++h) store_partial(a.end, split, h, live, row, col, v[h]);
    } else {
      finish<32>(a.end, live, row, col, v[0], v[kHalves - 1]);
    }
  }
}

// The tile shapes, by ProductPlan::tile.
template <bool kFp16, int kForm, int kHalves>
hipError_t launch_tile(int tile, ProductArgs& a, hipStream_t stream) {
  const int bm = kTileM[tile], bn = kTileN[tile] / (kHalves == 2 ? 2 : 1);
  a.tiles_m = (int32_t)((a.end.rows + bm - 1) / bm);
  a.tiles_n = (int32_t)((a.end.cols + bn - 1) / bn);
  const int64_t blocks = (int64_t)a.tiles_m * a.tiles_n * a.splits;
  if (blocks < 1 || blocks > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  switch (tile) {
    case 0: return launch_kernel(product_kernel<kFp16, kForm, kHalves, 256, 256, 2, 4>, grid, dim3(512), 0, stream, a);
    case 1: return launch_kernel(product_kernel<kFp16, kForm, kHalves, 128, 128, 2, 2>, grid, dim3(256), 0, stream, a);
    case 2: return launch_kernel(product_kernel<kFp16, kForm, kHalves, 64, 128, 2, 2>, grid, dim3(256), 0, stream, a);
  }
  return hipErrorInvalidValue;
}

template <bool kFp16>
hipError_t launch(Form form, const ProductPlan& plan, ProductArgs& a, hipStream_t stream) {
  a.splits = plan.splits;
  const bool two = a.end.halves == 2;
  switch (form) {
    case kForward:
      return two ? launch_tile<kFp16, kForward, 2>(plan.tile, a, stream) : launch_tile<kFp16, kForward, 1>(plan.tile, a, stream);
    case kDx: return two ? hipErrorInvalidValue : launch_tile<kFp16, kDx, 1>(plan.tile, a, stream);
    case kDw:
      return two ? launch_tile<kFp16, kDw, 2>(plan.tile, a, stream) : launch_tile<kFp16, kDw, 1>(plan.tile, a, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace mm
}  // namespace pointid
