// Forward products of a few rows (serving): y = x w with the weights read once, every value
// multiplied in fp32 with that of each row.  Bound by the bytes of the weights: fp32 8192 x
// 8192, 1 row 55 us (4.9 TB/s), 4 rows 59, 8 rows 64; gated 104, 112 and 122 (5.2 to 4.4); bf16
// gated 4096 x 12288, 1 row 46 (4.4).
// The inner index is split over blocks until there are about 3 a CU, as one block's reads in
// flight do not fill the memory; the join adds their sums in order.
#include "internal.h"
#include "layers_end.h"

namespace pointid {
namespace {

constexpr int kStrip = 256;      // columns of a block
constexpr int kChunk = 512;      // inner indices whose x values are in shared memory at once

struct RowsArgs {
  Strided x;
  Strided w[2];
  int64_t inner;
  int64_t per_split;             // inner indices of a split
  End end;
};

// A wave reads 256 columns of kRowsPer rows of the weights at a time, 16 bytes a lane (long
// stretches of a row: 64 columns took a third more time at 4 rows), the next reads under way
// while it multiplies; the block's 4 waves take turns along the inner index.  The lanes of a
// column are added in a fixed order at the end: lanes, then waves, then (elsewhere) splits.
template <int kM, int kType, int kHalves>
__global__ void __launch_bounds__(256) rows_kernel(RowsArgs a) {
  constexpr int kCols = kType == POINTID_FP32 ? 4 : 8;                  // of a lane
  constexpr int kLanes = kStrip / kCols;
  constexpr int kRowsPer = 64 / kLanes;
  constexpr int kStep = 4 * kRowsPer;
  constexpr int kAhead = kHalves == 2 ? 2 : 4;          // reads of a half in flight a lane, and as many again
  __shared__ float xs[(kChunk + 1) * kM];               // and a row of zeros, for what is past the end
  __shared__ float cs[kHalves][kM][kStrip];
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int64_t col0 = (int64_t)blockIdx.x * kStrip;
  const int64_t col = col0 + lane % kLanes * kCols;
  const int64_t first = a.per_split * blockIdx.y;
  const int64_t last = first + a.per_split < a.inner ? first + a.per_split : a.inner;
  float acc[kHalves][kM][kCols] = {};
  if (tid < kM) xs[kChunk * kM + tid] = 0.f;

  // A lane whose columns do not all exist reads the row's last ones instead (cols >= kCols).
  constexpr int kSize = kType == POINTID_FP32 ? 4 : 2;
  constexpr uint32_t kNowhere = 0x80000000u;           // past the resource's range: reads 0
  const int64_t from = col < a.end.cols - kCols ? col : a.end.cols - kCols;
  const int64_t origin = col0 < a.end.cols - kCols ? col0 : a.end.cols - kCols;      // the first of any lane's
  const char* wp[kHalves];
  uint32_t offset[kHalves], step[kHalves];
#pragma unroll
  for (int h = 0; h < kHalves; ++h) {
    const int64_t pitch = a.w[h].sk * kSize;
    wp[h] = static_cast<const char*>(a.w[h].p) + (first + wave * kRowsPer) * pitch + origin * kSize;
    offset[h] = (uint32_t)((lane / kLanes) * pitch + (from - origin) * kSize);
    step[h] = (uint32_t)(kStep * pitch);
  }
  auto values = [](const uint4& r, float* w) {
    const uint32_t v[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kSize == 4) {
        w[i] = __uint_as_float(v[i]);
      } else {
        w[2 * i] = from16((uint16_t)v[i], kType);
        w[2 * i + 1] = from16((uint16_t)(v[i] >> 16), kType);
      }
    }
  };
  for (int64_t k0 = first; k0 < last; k0 += kChunk) {
    const int len = (int)(last - k0 < kChunk ? last - k0 : kChunk);
    __syncthreads();
    for (int i = tid; i < len * kM; i += 256) {
      const int r = i / len, k = i - r * len;
      xs[k * kM + r] = r < a.end.rows ? load_any(a.x.p, r * a.x.si + k0 + k, kType) : 0.f;
    }
    __syncthreads();
    // turns of kAhead reads: those of the next turn are under way while this one multiplies
    const int mine = wave * kRowsPer + lane / kLanes;
    uint4 raw[2][kHalves][kAhead];
    auto fetch = [&](int buf, int base) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int k = base + u * kStep;
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
          const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
              const_cast<char*>(wp[h]), (short)0, (int)kNowhere, 0x00020000);
          raw[buf][h][u] = __builtin_bit_cast(
              uint4, __builtin_amdgcn_raw_buffer_load_b128(r, k < len ? offset[h] : kNowhere, u * step[h], 0));
        }
      }
#pragma unroll
      for (int h = 0; h < kHalves; ++h) wp[h] += (int64_t)kAhead * step[h];
    };
    auto multiply = [&](int buf, int base) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int k = base + u * kStep < len ? base + u * kStep : kChunk;
        float x[kM];
#pragma unroll
        for (int r = 0; r < kM; ++r) x[r] = xs[k * kM + r];
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
          float w[kCols];
          values(raw[buf][h][u], w);
#pragma unroll
          for (int r = 0; r < kM; ++r)
#pragma unroll
            for (int c = 0; c < kCols; ++c) acc[h][r][c] += x[r] * w[c];
        }
      }
    };
    constexpr int kTurn = kStep * kAhead;
    const char* at[kHalves];
#pragma unroll
    for (int h = 0; h < kHalves; ++h) at[h] = wp[h];
    fetch(0, mine);
    for (int base = mine; base - mine < len; base += 2 * kTurn) {
      fetch(1, base + kTurn);
      multiply(0, base);
      if (base + kTurn - mine >= len) break;
      fetch(0, base + 2 * kTurn);
      multiply(1, base + kTurn);
    }
#pragma unroll
    for (int h = 0; h < kHalves; ++h) wp[h] = at[h] + (int64_t)(kChunk / kStep) * step[h];
  }
#pragma unroll
  for (int h = 0; h < kHalves; ++h)
#pragma unroll
    for (int r = 0; r < kM; ++r)
#pragma unroll
      for (int c = 0; c < kCols; ++c)
#pragma unroll
        for (int x = kLanes; x < 64; x *= 2) acc[h][r][c] += __shfl_xor(acc[h][r][c], x, 64);
  for (int turn = 0; turn < 4; ++turn) {
    if (wave == turn && lane < kLanes) {
#pragma unroll
      for (int h = 0; h < kHalves; ++h)
#pragma unroll
        for (int r = 0; r < kM; ++r)
#pragma unroll
          for (int c = 0; c < kCols; ++c) {
            if (from + c < col) continue;              // the lane before has it
            float* const p = &cs[h][r][from + c - col0];
            *p = turn == 0 ? acc[h][r][c] : *p + acc[h][r][c];
          }
    }
    __syncthreads();
  }
  // 8 columns of a row a lane, whole waves at a time
  constexpr int kUnits = kStrip / 8;
  for (int i = tid; i < (kM * kUnits + 63) / 64 * 64; i += 256) {
    const int row = i / kUnits, unit = i % kUnits, r = row < kM ? row : 0;
    const int64_t at = col0 + unit * 8;
    const bool here = row < kM && row < a.end.rows, live = here && at < a.end.cols;
    float v[kHalves][8];
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
      for (int c = 0; c < 8; ++c) v[h][c] = cs[h][r][unit * 8 + c];
    if (a.end.mode == kEndPartial) {
#pragma unroll
      for (int h = 0; h < kHalves; ++h) store_partial(a.end, blockIdx.y, h, here, row, at, v[h]);
    } else {
      float bias[2][8];
      load_bias(a.end.bias0, at, a.end.cols, bias[0]);
      load_bias(a.end.bias1, at, a.end.cols, bias[1]);
      const int count = piece_cols(a.end.cols, at);
      Residual<kType> residual;
      residual.load(residual.at(a.end, r, at), a.end.residual && live ? count : 0);
      Targets<kType, kHalves> to;
      to.init(a.end, r, at);
      finish<kType, kHalves>(a.end, to, live, at % kBlock8 == 0, count, v[0], v[kHalves - 1], bias[0], bias[1], residual,
                              1.f);
    }
  }
}

template <int kM, int kHalves>
hipError_t launch_type(const RowsArgs& a, dim3 grid, hipStream_t stream) {
  switch (a.w[0].dtype) {
    case POINTID_FP32: return launch_kernel(rows_kernel<kM, POINTID_FP32, kHalves>, grid, dim3(256), 0, stream, a);
    case POINTID_BF16: return launch_kernel(rows_kernel<kM, POINTID_BF16, kHalves>, grid, dim3(256), 0, stream, a);
  }
  return launch_kernel(rows_kernel<kM, POINTID_FP16, kHalves>, grid, dim3(256), 0, stream, a);
}

template <int kHalves>
hipError_t launch_rows(const RowsArgs& a, dim3 grid, hipStream_t stream) {
  if (a.end.rows <= 1) return launch_type<1, kHalves>(a, grid, stream);
  if (a.end.rows <= 2) return launch_type<2, kHalves>(a, grid, stream);
  if (a.end.rows <= 4) return launch_type<4, kHalves>(a, grid, stream);
  return launch_type<8, kHalves>(a, grid, stream);
}

int64_t rows_per_split(int64_t inner, int splits) { return ((inner + splits - 1) / splits + 7) / 8 * 8; }

}  // namespace

// About 3 blocks a CU, each over at least 64 inner indices.
int few_rows_splits(int64_t inner, int64_t cols, int halves, int cus) {
  const int64_t strips = (cols + kStrip - 1) / kStrip;
  int64_t s = 3 * (int64_t)cus / strips, most = (inner + 63) / 64;
  s = s < 1 ? 1 : s;
  s = s > most ? most : s;
  s = s > 4096 ? 4096 : s;
  const int64_t per = rows_per_split(inner, (int)s);
  return (int)((inner + per - 1) / per);               // no split without work
}

hipError_t launch_layers_rows(const Strided& x, const Strided* w, int64_t inner, const End& end, int splits,
                              hipStream_t stream) {
  if (end.rows < 1 || end.rows > kFewRows || splits < 1 || splits > 65535) return hipErrorInvalidValue;
  RowsArgs a;
  a.x = x;
  a.w[0] = w[0];
  a.w[1] = w[end.halves == 2 ? 1 : 0];
  a.inner = inner;
  a.per_split = rows_per_split(inner, splits);
  a.end = end;
  const dim3 grid((unsigned)((end.cols + kStrip - 1) / kStrip), (unsigned)splits);
  return end.halves == 2 ? launch_rows<2>(a, grid, stream) : launch_rows<1>(a, grid, stream);
}

}  // namespace pointid
