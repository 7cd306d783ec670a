// Products on the matrix cores (16-bit operands, fp32 sums), one template for the three
// forms of layers.h: x w, dz w^T and x^T dz, the sums over k, n and m.
//
// A block computes kBM x kBN results with 16x16x32 MFMAs (a loop of these alone runs at
// 2.0 PFLOP/s on random bf16 values, one of 32x32x16 at 1.8: the card is at its power limit,
// and they pass half as many sums per multiplication through the registers).  Both
// operands go through shared memory, 64 inner indices at a time, two stages (three for a
// tile that a CU holds once and whose multiplications are shorter than the loads' latency),
// written by loads that go there directly (16 bytes a lane).  An operand whose rows run
// along the inner index (x and dz of dx and forward's x) is read as fragments with 16-byte
// reads; one whose rows are indexed by the inner index (W of the forward form, both of dW)
// with the transposing read, 4 x 16 values at a time, so no form needs a transposed copy.
//
// Bound by power where there is work for all CUs: 16384 x 4096 x 4096 in bf16 407 us, 1.35
// PFLOP/s (with GELU and a residual 458), MFMA 55-65 % busy at 1.9 GHz; 8192 x 16384 x 4096
// 832 us, its dx 826, its dW 874; a gated 8192 x 4096 x 8192 824, 892 with g and u kept in 8
// bits.  Few rows are bound by the bytes of the weights: 4 rows of a gated 4096 x 12288
// 51 us with the join, 4.0 TB/s.
//
// The results come out with the right operand as the MFMA's first, so a lane holds 4
// consecutive columns of one row at a time; the end passes them through shared memory to
// where 8 lanes hold 64 columns of a row (two halves: 4 lanes 32 columns of both).
//
// Pieces of 16 bytes stand in shared memory in a permuted order that the loads apply to
// their global addresses.  Rows of 64 inner indices (128 bytes): piece p of row r at
// p ^ (r / 2 % 8), so that 16 lanes reading one piece of 16 rows touch all banks (rows of
// 32 inner indices, in the fp32 kernel: p ^ (-(r / 4) % 4); without the minus lanes 0-3 and
// 12-15 met 20-27, which are served with them: 0.22 to 0.36 of the cycles).  Rows of columns:
// the pair of pieces g of row r at g ^ (r % 4 + 4 (r / 8 % 2)) (rows of 128 bytes: g ^ (r / 2
// % 2 + 2 (r / 8 % 2)), of 64: g ^ (r / 8 % 2)), so that the rows r .. r + 3 and r + 8 ..
// r + 11 of 16 columns that 32 lanes of a transposing read take do.
#pragma once

#include "internal.h"
#include "layers_end.h"

namespace pointid {
namespace mm {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

constexpr int kBK = 64;                     // inner indices of a stage
constexpr uint32_t kNowhere = 0x80000000u;  // an offset past the resource's range: reads 0

// The piece's place in a row of kPieces pieces of 16 bytes; kInner: rows along the inner index.
template <bool kInner, int kPieces>
__device__ __forceinline__ int place(int row, int piece) {
  if constexpr (kInner) return kPieces == 8 ? piece ^ ((row >> 1) & 7) : piece ^ (-(row >> 2) & 3);
  if constexpr (kPieces >= 16) return piece ^ (((row & 3) | (row >> 1 & 4)) << 1);
  if constexpr (kPieces == 4) return piece ^ (row >> 3 & 1) << 1;
  return piece ^ (((row >> 1 & 1) | (row >> 2 & 2)) << 1);
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
               :: "s"(lds), "v"(offset), "s"(rsrc) : "memory", "m0");
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
  int inner;                                // first inner index of the first piece
  // ... and of piece i: the same, or as many rows on
  static constexpr int kStep = kInner ? 0 : kThreads / kPieces;
  static_assert(!kInner || kThreads / kPieces % 16 == 0, "the places repeat");

  // side0: the tile's first row or column of `sides`
  __device__ __forceinline__ void init(int tid, int64_t side0, int64_t sides, int64_t ld) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = i * kThreads + tid, row = at / kPieces;
      const int piece = place<kInner, kPieces>(row, at % kPieces);       // its own inverse
      const int side = kInner ? row : piece * 8;
      if (i == 0) inner = kInner ? piece * 8 : row;
      offset[i] = side0 + side < sides ? (uint32_t)((row * ld + piece * 8) * 2) : kNowhere;
    }
  }
  // Load i of the stage at `from`, `left` inner indices of it there.
  __device__ __forceinline__ void load(int i, intx4 from, int left, uint32_t lds, int wave) const {
    load_to_lds(from, inner + i * kStep < left ? offset[i] : kNowhere, lds + (i * kThreads + wave * 64) * 16);
  }
};

// Fragments: 8 consecutive inner indices of one row or column a lane (lane % 16; the next 16
// lanes the next 8).  kInner: group i of 16 stands i * 16 rows on; else each group has an
// address of its own.
template <bool kInner, int kSide, int kFrags, int kInners = kBK>
struct Frags {
  static constexpr int kSteps = kInners / 32, kRow = kInners * 2;
  int base[kInner ? kSteps : kFrags];
  // side0(i, &tile): group i's first row or column, and the offset of its tile
  template <class F>
  __device__ __forceinline__ void init(int lane, F&& side0) {
    if constexpr (kInner) {
      int tile;
      const int row = side0(0, &tile) + lane % 16;
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        base[s] = tile + row * kRow + place<true, kInners / 8>(row, 4 * s + lane / 16) * 16;
    } else {
      // the lane's address in a read of 4 rows x 16 columns by 16 lanes
      const int row = lane / 16 * 8 + lane % 16 / 4;
#pragma unroll
      for (int i = 0; i < kFrags; ++i) {
        int tile;
        const int col = side0(i, &tile) + lane % 4 * 4;
        base[i] = tile + row * (kSide * 2) + place<false, kSide / 8>(row, col / 8) * 16 + col % 8 * 2;
      }
    }
  }
  // inner indices 32 s .. 32 s + 31 of group i
  __device__ __forceinline__ uint4 read(const char* tile, int i, int s) const {
    if constexpr (kInner) {
      return *reinterpret_cast<const uint4*>(tile + base[s] + i * 16 * kRow);
    } else {
      typedef __attribute__((address_space(3))) shortx4 LdsShort4;
      const char* p = tile + base[i] + s * 32 * kSide * 2;
      const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4*)p);
      const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4*)(p + 4 * kSide * 2));
      const uint2 l = __builtin_bit_cast(uint2, lo), h = __builtin_bit_cast(uint2, hi);
      return make_uint4(l.x, l.y, h.x, h.y);
    }
  }
};

// All reads of this wave from shared memory and all but its newest kCount loads into it done,
// then the block's barrier.  The reads' wait is the compiler's own instruction, so that it
// does not wait for them again afterwards; of the loads it knows nothing.
template <int kCount>
__device__ __forceinline__ void stage_ready() {
  static_assert(kCount < 64, "the counter's range");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);                    // lgkmcnt(0)
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kCount) : "memory");
}

// The block's tile and split.
struct Place {
  uint32_t split;
  int64_t tm, tn;
};
__device__ __forceinline__ Place block_place(const ProductArgs& a, uint32_t block) {
  // Blocks go to the 8 XCDs in turn: each XCD takes a contiguous stretch of the tiles, in
  // groups of 8 rows of tiles walked column by column, so that the blocks which run
  // together on an XCD share operands in its L2.
  const uint32_t xcd = block % 8;
  uint32_t id = xcd * a.xcd_each + (xcd < (uint32_t)a.xcd_more ? xcd : a.xcd_more) + block / 8;
  uint32_t split = 0;
  if (a.splits > 1) {
    const uint32_t tiles = (uint32_t)a.tiles_m * a.tiles_n;
    split = id / tiles;
    id -= split * tiles;
  }
  constexpr uint32_t kGroup = 8;
  const uint32_t group = id / (kGroup * a.tiles_n), in = id - group * kGroup * a.tiles_n;
  const uint32_t rows_here = a.tiles_m - group * kGroup < kGroup ? a.tiles_m - group * kGroup : kGroup;
  const uint32_t tn = in / rows_here;
  return {split, group * kGroup + (in - tn * rows_here), tn};
}

// The end of a wave's results (bias, activation, product of the halves, residual and kept
// activations are done here, on the sums in registers: as a pass of its own the GELU and
// residual of 16384 x 4096 would move 400 MB more, 85 us).  Rows from `row0` of kFragsM groups of 16, columns from `col0`
// (of each half).  One copy of the end's code: 32 rows x 64 columns a turn (two halves: 32
// columns of each) through the wave's kEndWave bytes of shared memory, from a lane's 4
// columns of one row to 16 bytes and more a lane along the rows.  The residual of a turn is
// read a turn ahead.
constexpr int kEndPitch = 64 + 4;
constexpr int kEndWave = 32 * kEndPitch * 4;
template <int kType, int kHalves, int kFragsM>
__device__ __forceinline__ void end_tile(const End& e, const floatx4 (&acc)[kFragsM][4], float* es, int lane, int split,
                                         int64_t row0, int64_t col0, float unscale) {
  constexpr int kLanes = kHalves == 2 ? 4 : 8;           // of a row
  constexpr int kSteps = kLanes / 2, kRows = 64 / kLanes, kTurns = (kFragsM + 1) / 2;
  const int64_t col = col0 + lane % kLanes * 8;
  const int n = piece_cols(e.cols, col);
  row0 += lane / kLanes;
  // rows of the result from the lane's first on
  int left = (int)(e.rows - row0 < kFragsM * 16 ? e.rows - row0 : kFragsM * 16);
  const float* const from = es + lane / kLanes * kEndPitch + lane % kLanes * 8;
  float* const into = es + lane % 16 * kEndPitch + lane / 16 * 4;
  auto pass = [&](const floatx4(&c)[2][4]) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<floatx4*>(into + i / 4 * 16 * kEndPitch + i % 4 * 16) = c[i / 4][i % 4];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  auto take = [&](int s, float(&v)[kHalves][8]) {
#pragma unroll
    for (int h = 0; h < kHalves; ++h) __builtin_memcpy(v[h], from + s * kRows * kEndPitch + h * 32, 32);
  };
  auto sums = [&](int turn, floatx4(&c)[2][4]) {
    static_for<kTurns>([&](auto t) {
      if (turn == t)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (2 * t + i / 4 < kFragsM) c[i / 4][i % 4] = acc[2 * t + i / 4 < kFragsM ? 2 * t + i / 4 : 0][i % 4];
    });
  };
  if (e.mode == kEndPartial) {
#pragma nounroll
    for (int turn = 0; turn < kTurns; ++turn, row0 += 32, left -= 32) {
      floatx4 c[2][4] = {};
      sums(turn, c);
      pass(c);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        float v[kHalves][8];
        take(s, v);
#pragma unroll
        for (int h = 0; h < kHalves; ++h) store_partial(e, split, h, s * kRows < left, row0 + s * kRows, col, v[h]);
      }
    }
    return;
  }
  float b0[8], b1[8];
  if (e.mode != kEndStore) {
    load_bias(e.bias0, col, e.cols, b0);
    if constexpr (kHalves == 2) load_bias(e.bias1, col, e.cols, b1);
  }
  Targets<kType, kHalves> to;
  to.init(e, row0, col);
  const bool add = kHalves == 1 && e.residual;
  const char* residual = add ? Residual<kType>::at(e, row0, col) : nullptr;
  const int64_t residual_step = kRows * e.ld_residual * (kType == POINTID_FP32 ? 4 : 2);
  Residual<kType> next[kSteps];
  auto read = [&](int rows) {
    if (!add) return;
#pragma unroll
    for (int s = 0; s < kSteps; ++s, residual += residual_step) next[s].load(residual, s * kRows < rows ? n : 0);
  };
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
#pragma unroll
    for (uint32_t& w : next[s].w) w = 0;
  read(left);
#pragma nounroll
  for (int turn = 0; turn < kTurns; ++turn) {
    floatx4 c[2][4] = {};
    sums(turn, c);
    Residual<kType> now[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) now[s] = next[s];
    if (turn + 1 < kTurns) read(left - 32);
    pass(c);
#pragma nounroll
    for (int s = 0; s < kSteps; ++s, left -= kRows) {
      float v[kHalves][8];
      take(s, v);
      Residual<kType> r = now[0];
      if (add)
        static_for<kSteps>([&](auto t) {
          if (s == t) r = now[t];
        });
      finish<kType, kHalves>(e, to, n > 0 && left > 0, lane % 4 == 0, n, v[0], v[kHalves - 1], b0, b1, r, unscale);
      to.down(e, kRows);
    }
  }
}

template <bool kFp16>
__device__ __forceinline__ floatx4 mfma(const uint4& a, const uint4& b, const floatx4& c) {
  return Op16<kFp16>::mfma(a, b, c);
}

// Shared memory of a block: its stages, where the end's takes their place, and a little more
// for that with many small waves.
template <int kBM, int kBN, int kWM, int kWN, int kStages>
constexpr int shared_bytes() {
  constexpr int kStage = (kBM + kBN) * kBK * 2;
  return kWM * kWN * kEndWave > kStages * kStage ? kWM * kWN * kEndWave : kStages * kStage;
}

template <bool kFp16, int kForm, int kHalves, int kBM, int kBN, int kWM, int kWN, int kStages>
__device__ __forceinline__ void product_block(const ProductArgs& a, uint32_t block, char* smem) {
  constexpr int kThreads = 64 * kWM * kWN;
  constexpr int kType = kFp16 ? POINTID_FP16 : POINTID_BF16;
  constexpr bool kLeftInner = kForm != kDw, kRightInner = kForm == kDx;
  static_assert(!kRightInner || kHalves == 1, "dx has one half");
  constexpr int kHN = kBN / 2;                           // columns of each half of the tile
  constexpr int kFragsM = kBM / kWM / 16, kFragsN = 4;
  static_assert(kBN / kWN == 64, "a wave takes 64 columns");
  using Left = Tile<kLeftInner, kBM, kThreads>;
  using Right = Tile<kRightInner, kHN, kThreads>;
  constexpr int kStage = Left::kBytes + 2 * Right::kBytes;
  constexpr int kStageLoads = Left::kLoads + 2 * Right::kLoads;

  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int wm = wave / kWN, wn = wave % kWN;

  // read here, as every block of a short sum would wait for it in its end (dx and dW of 1693 x
  // 92928 x 128, dz of silu: 228 us with that for 212)
  const float unscale = unscale_of<kType>(a.end);
  const Place at = block_place(a, block);
  const uint32_t split = at.split;
  const int64_t tm = at.tm, tn = at.tn;
  const int64_t row0 = tm * kBM;
  const int64_t col0 = tn * (kHalves == 2 ? kHN : kBN), col1 = kHalves == 2 ? col0 : col0 + kHN;
  Left left;
  Right right0, right1;
  left.init(tid, row0, a.end.rows, a.ld_left);
  right0.init(tid, col0, a.end.cols, a.ld_right);
  right1.init(tid, col1, a.end.cols, a.ld_right);
  // A wave's columns: with two halves 32 of each; with one, 64 side by side (they lie in
  // one half of the tile).
  Frags<kLeftInner, kBM, kFragsM> lf;
  Frags<kRightInner, kHN, kFragsN> rf;
  lf.init(lane, [&](int i, int* tile) {
    *tile = 0;
    return wm * (kBM / kWM) + 16 * i;
  });
  rf.init(lane, [&](int i, int* tile) {
    const int half = kHalves == 2 ? i / 2 : wn * 64 / kHN;
    *tile = Left::kBytes + half * Right::kBytes;
    return kHalves == 2 ? wn * 32 + i % 2 * 16 : wn * 64 % kHN + 16 * i;
  });

  // the split's stages, and where the next one to load is
  int to_load = a.split_each + (split < (uint32_t)a.split_more);
  const uint32_t first = split * a.split_each + (split < (uint32_t)a.split_more ? split : a.split_more);
  int term = 0;
  if (a.splits > 1) term = (int)(first / (uint32_t)a.stages);
  int k0 = (int)(first - (uint32_t)term * a.stages) * kBK;
  const int stages = to_load;
  const int64_t left_step = (kLeftInner ? kBK : kBK * a.ld_left) * 2;
  const int64_t right_step = (kRightInner ? kBK : kBK * a.ld_right) * 2;
  const int64_t left_at = (kLeftInner ? row0 * a.ld_left : row0) * 2;
  const int64_t right_at0 = (kRightInner ? col0 * a.ld_right : col0) * 2;
  const int64_t right_at1 = (kRightInner ? col1 * a.ld_right : col1) * 2;
  const char *lp, *rp0, *rp1;
  auto enter = [&](int k) {
    const Term& t = a.term[term];
    const int64_t s = k / kBK;
    lp = static_cast<const char*>(t.left) + left_at + s * left_step;
    rp0 = static_cast<const char*>(t.right0) + right_at0 + s * right_step;
    rp1 = static_cast<const char*>(kHalves == 2 ? t.right1 : t.right0) + right_at1 + s * right_step;
  };
  enter(k0);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;

  // part q of kParts of the loads of the next stage (a compile-time constant)
  constexpr int kParts = kFragsM / 2;
  auto issue = [&](auto q, int stage) {
    constexpr int kLoads = kStageLoads;
    const uint32_t to = lds0 + stage * kStage;
    const int left_of = a.inner - k0;
    static_for<kLoads>([&](auto n) {
      if constexpr (n * kParts / kLoads == q) {
        if constexpr (n < Left::kLoads)
          left.load(n, resource(lp), left_of, to, wave);
        else if constexpr (n < Left::kLoads + Right::kLoads)
          right0.load(n - Left::kLoads, resource(rp0), left_of, to + Left::kBytes, wave);
        else
          right1.load(n - Left::kLoads - Right::kLoads, resource(rp1), left_of, to + Left::kBytes + Right::kBytes, wave);
      }
    });
    if constexpr (q == kParts - 1) {
      k0 += kBK;
      lp += left_step, rp0 += right_step, rp1 += right_step;
      if (k0 >= a.inner && --to_load > 0) {
        k0 = 0;
        ++term;
        enter(0);
      } else if (k0 < a.inner) {
        --to_load;
      }
    }
  };

  // A stage is multiplied in 4 turns, 32 inner indices by half of the wave's rows; the
  // fragments of a turn are read while the turn before multiplies.  The last turn multiplies
  // after the barrier that makes the next stage ready and this one free, so that the next
  // stage's first fragments and the loads of the stage after it are under way meanwhile.
  floatx4 acc[kFragsM][kFragsN] = {};
  uint4 l[2][kParts], r[2][kFragsN];
  auto read_left = [&](int turn, const char* tile) {
#pragma unroll
    for (int i = 0; i < kParts; ++i) l[turn % 2][i] = lf.read(tile, turn % 2 * kParts + i, turn / 2);
  };
  auto read_right = [&](int s, const char* tile) {
#pragma unroll
    for (int j = 0; j < kFragsN; ++j) r[s][j] = rf.read(tile, j, s);
  };
  auto multiply = [&](int turn, int i) {
    floatx4(&c)[kFragsN] = acc[turn % 2 * kParts + i];
#pragma unroll
    for (int j = 0; j < kFragsN; ++j) c[j] = mfma<kFp16>(r[turn / 2][j], l[turn % 2][i], c[j]);
  };
  if (stages > 0) {
    static_for<kStages>([&](auto n) {
      if (n < stages) static_for<kParts>([&](auto q) { issue(q, n); });
    });
    if (stages >= kStages)
      stage_ready<(kStages - 1) * kStageLoads>();
    else
      stage_ready<0>();
    read_right(0, smem);
    read_left(0, smem);
    int stage = 0;
    for (int it = stages; it > 0; --it) {
      const char* tile = smem + stage * kStage;
#pragma unroll
      for (int turn = 0; turn < 3; ++turn) {
        if (turn == 1) read_right(1, tile);
        read_left(turn + 1, tile);
#pragma unroll
        for (int i = 0; i < kParts; ++i) multiply(turn, i);
        __builtin_amdgcn_sched_barrier(0);
      }
      // the next stage: all that is newer may still be under way, as long as that is kStages - 2
      if (kStages > 2 && it >= kStages)
        stage_ready<(kStages - 2) * kStageLoads>();
      else
        stage_ready<0>();
      const int after = stage + 1 < kStages ? stage + 1 : 0;
      if (it > 1) {
        const char* next = smem + after * kStage;
        read_right(0, next);
        read_left(0, next);
      }
      const bool more = to_load > 0;
      static_for<kParts>([&](auto q) {
        __builtin_amdgcn_sched_barrier(0);
        multiply(3, q);
        __builtin_amdgcn_sched_barrier(0);
        if (more) issue(q, stage);
      });
      stage = after;
    }
  }
  stage_ready<0>();                                      // the stages are free for the end

  end_tile<kType, kHalves, kFragsM>(a.end, acc, reinterpret_cast<float*>(smem) + wave * kEndWave / 4, lane, split,
                                             row0 + wm * (kBM / kWM),
                                             col0 + wn * (kHalves == 2 ? 32 : 64), unscale);
}

template <bool kFp16, int kForm, int kHalves, int kBM, int kBN, int kWM, int kWN, int kStages>
__global__ void __launch_bounds__(64 * kWM * kWN) product_kernel(ProductArgs a) {
  __shared__ __align__(1024) char smem[shared_bytes<kBM, kBN, kWM, kWN, kStages>()];
  product_block<kFp16, kForm, kHalves, kBM, kBN, kWM, kWN, kStages>(a, blockIdx.x, smem);
}

// Both products of a gradient in one launch, their blocks mixed in units of 8 (one of each
// XCD).  Those with the longer sums come first: their units are spread evenly over the first
// half of the launch.  The very first blocks take the column sums.
struct PairArgs {
  ProductArgs dx, dw;
  SumsJobs sums;
  uint32_t sums_blocks, sums_units;
  int32_t dx_first;
  uint32_t first_units;
  uint64_t ratio;              // 2^32 times their share of that part
};
// The block's part: dx(args, block) or dw(args, block), or column sums in `smem`.
template <int kThreads, class Dx, class Dw>
__device__ __forceinline__ void pair_block(const PairArgs& a, char* smem, Dx&& dx, Dw&& dw) {
  if (blockIdx.x < a.sums_units * 8) {
    if (blockIdx.x < a.sums_blocks) sum_columns<kThreads>(a.sums, blockIdx.x, reinterpret_cast<float*>(smem));
    return;
  }
  const uint32_t unit = blockIdx.x / 8 - a.sums_units, xcd = blockIdx.x % 8;
  auto first_before = [&](uint32_t u) {
    const uint64_t n = u * a.ratio >> 32;
    return n < a.first_units ? (uint32_t)n : a.first_units;
  };
  const uint32_t before = first_before(unit);
  const bool first = first_before(unit + 1) > before;
  const uint32_t mine = first ? before : unit - before;    // the block's unit of its product
  auto here = [&](const ProductArgs& p) { return mine < p.xcd_each + (xcd < (uint32_t)p.xcd_more ? 1u : 0u); };
  if (first == (a.dx_first != 0)) {
    if (here(a.dx)) dx(a.dx, mine * 8 + xcd);
  } else {
    if (here(a.dw)) dw(a.dw, mine * 8 + xcd);
  }
}
template <bool kFp16, int kHalves, int kBM, int kBN, int kWM, int kWN, int kStages>
__global__ void __launch_bounds__(64 * kWM * kWN) pair_kernel(PairArgs a) {
  __shared__ __align__(1024) char smem[shared_bytes<kBM, kBN, kWM, kWN, kStages>()];
  pair_block<64 * kWM * kWN>(
      a, smem,
      [&](const ProductArgs& p, uint32_t block) { product_block<kFp16, kDx, 1, kBM, kBN, kWM, kWN, kStages>(p, block, smem); },
      [&](const ProductArgs& p, uint32_t block) {
        product_block<kFp16, kDw, kHalves, kBM, kBN, kWM, kWN, kStages>(p, block, smem);
      });
}

// What a launch works out for its blocks; returns their number, or 0.
inline int64_t spread(ProductArgs& a, int64_t rows, int64_t cols, int inners) {
  const int64_t tm = (a.end.rows + rows - 1) / rows, tn = (a.end.cols + cols - 1) / cols;
  if (tm < 1 || tn < 1 || a.splits < 1 || a.terms < 1 || tm > INT32_MAX / tn || tm * tn > INT32_MAX / a.splits) return 0;
  a.tiles_m = (int32_t)tm;
  a.tiles_n = (int32_t)tn;
  const int64_t blocks = tm * tn * a.splits;
  a.xcd_each = (int32_t)(blocks / 8);
  a.xcd_more = (int32_t)(blocks % 8);
  a.stages = (int32_t)(((int64_t)a.inner + inners - 1) / inners);
  const int64_t total = (int64_t)a.stages * a.terms;
  a.split_each = (int32_t)(total / a.splits);
  a.split_more = (int32_t)(total % a.splits);
  return blocks;
}

// The tile shapes, by ProductPlan::tile.
template <bool kFp16, int kForm, int kHalves>
hipError_t launch_tile(int tile, ProductArgs& a, hipStream_t stream) {
  const int bm = kTileM[tile], bn = kTileN[tile] / (kHalves == 2 ? 2 : 1);
  const int64_t blocks = spread(a, bm, bn, kBK);
  if (blocks < 1 || a.end.dtype != (kFp16 ? POINTID_FP16 : POINTID_BF16)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  switch (tile) {
    case 0: return launch_kernel(product_kernel<kFp16, kForm, kHalves, 256, 256, 2, 4, 2>, grid, dim3(512), 0, stream, a);
    case 1: return launch_kernel(product_kernel<kFp16, kForm, kHalves, 128, 128, 4, 2, 3>, grid, dim3(512), 0, stream, a);
    case 2: return launch_kernel(product_kernel<kFp16, kForm, kHalves, 128, 128, 4, 2, 2>, grid, dim3(512), 0, stream, a);
    case 3: return launch_kernel(product_kernel<kFp16, kForm, kHalves, 64, 128, 2, 2, 2>, grid, dim3(256), 0, stream, a);
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

// The same of a pair of products in bm x bn tiles.
inline int64_t spread_pair(PairArgs& a, int64_t bm, int64_t bn, int inners) {
  const int64_t dx = spread(a.dx, bm, bn, inners), dw = spread(a.dw, bm, bn / a.dw.end.halves, inners);
  const uint64_t dx_units = (uint64_t)(dx + 7) / 8, dw_units = (uint64_t)(dw + 7) / 8, units = dx_units + dw_units;
  if (dx < 1 || dw < 1 || units > INT32_MAX / 16) return 0;
  a.dx_first = a.dx.split_each >= a.dw.split_each;
  const uint64_t first = a.dx_first ? dx_units : dw_units, part = first > units / 2 ? first : units / 2;
  a.first_units = (uint32_t)first;
  a.ratio = ((first << 32) + part - 1) / part;
  a.sums_blocks = a.sums.part ? a.sums.blocks() : 0;
  a.sums_units = (a.sums_blocks + 7) / 8;
  return (int64_t)(units + a.sums_units) * 8;
}

template <bool kFp16, int kHalves>
hipError_t launch_pair_tile(int tile, PairArgs& a, hipStream_t stream) {
  const int64_t blocks = spread_pair(a, kTileM[tile], kTileN[tile], kBK);
  constexpr int kType = kFp16 ? POINTID_FP16 : POINTID_BF16;
  if (blocks < 1 || a.dx.end.dtype != kType || a.dw.end.dtype != kType) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  switch (tile) {
    case 1: return launch_kernel(pair_kernel<kFp16, kHalves, 128, 128, 4, 2, 3>, grid, dim3(512), 0, stream, a);
    case 2: return launch_kernel(pair_kernel<kFp16, kHalves, 128, 128, 4, 2, 2>, grid, dim3(512), 0, stream, a);
    case 3: return launch_kernel(pair_kernel<kFp16, kHalves, 64, 128, 2, 2, 2>, grid, dim3(256), 0, stream, a);
  }
  return hipErrorInvalidValue;
}
template <bool kFp16>
hipError_t launch_pair(int tile, const ProductArgs& dx, const ProductArgs& dw, const SumsJobs& sums, hipStream_t stream) {
  PairArgs a;
  a.dx = dx, a.dw = dw, a.sums = sums;
  return dw.end.halves == 2 ? launch_pair_tile<kFp16, 2>(tile, a, stream) : launch_pair_tile<kFp16, 1>(tile, a, stream);
}

}  // namespace mm
}  // namespace pointid
