// Forward products of a few rows (serving): the weights are read once, every value
// multiplied in fp32 with that of each row.  Bound by the bytes of the weights.
#include "internal.h"
#include "layers_end.h"

namespace pointid {
namespace {

constexpr int kStrip = 64;       // columns of a block
constexpr int kChunk = 1024;     // inner indices whose x values are in shared memory at once

struct RowsArgs {
  Strided x;
  Strided w[2];
  int64_t inner;
  int64_t per_split;             // inner indices of a split, a multiple of 32
  End end;
};

// A wave reads kRowsPer rows of 64 columns of the weights at a time, 16 bytes a lane; the
// block's 4 waves take turns along the inner index.  The lanes of a column are added in a
// fixed order at the end: lanes, then waves, then (elsewhere) splits.
template <int kM, int kType, int kHalves>
__global__ void __launch_bounds__(256) rows_kernel(RowsArgs a) {
  constexpr int kCols = kType == POINTID_FP32 ? 4 : 8;                  // of a lane
  constexpr int kLanes = kStrip / kCols;
  constexpr int kRowsPer = 64 / kLanes;
  constexpr int kStep = 4 * kRowsPer;
  constexpr int kAhead = kHalves == 2 ? 4 : 8;         // reads in flight a lane
  __shared__ float xs[kChunk * kM];
  __shared__ float cs[4][kHalves][kM][kStrip];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int64_t col0 = (int64_t)blockIdx.x * kStrip;
  const int64_t col = col0 + lane % kLanes * kCols, n = a.end.cols - col;
  const int64_t first = a.per_split * blockIdx.y;
  const int64_t last = first + a.per_split < a.inner ? first + a.per_split : a.inner;
  float acc[kHalves][kM][kCols] = {};

  for (int64_t k0 = first; k0 < last; k0 += kChunk) {
    const int len = (int)(last - k0 < kChunk ? last - k0 : kChunk);
    __syncthreads();
    for (int i = tid; i < len * kM; i += 256) {
      const int r = i / len, k = i - r * len;
      xs[k * kM + r] = r < a.end.rows ? load_any(a.x.p, r * a.x.si + k0 + k, a.x.dtype) : 0.f;
    }
    __syncthreads();
    for (int base = wave * kRowsPer + lane / kLanes; base - lane / kLanes < len; base += kStep * kAhead) {
      float w[kHalves][kAhead][kCols];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int k = base + u * kStep;
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
          load_cols<kCols>(a.w[h].p, (k0 + k) * a.w[h].sk + col, kType,
                           k < len ? n : 0, w[h][u]);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int k = base + u * kStep;
        if (k >= len) continue;
#pragma unroll
        for (int r = 0; r < kM; ++r) {
          const float x = xs[k * kM + r];
#pragma unroll
          for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int c = 0; c < kCols; ++c) acc[h][r][c] += x * w[h][u][c];
        }
      }
    }
  }
#pragma unroll
  for (int h = 0; h < kHalves; ++h)
#pragma unroll
    for (int r = 0; r < kM; ++r)
#pragma unroll
      for (int c = 0; c < kCols; ++c) {
        float t = acc[h][r][c];
#pragma unroll
        for (int x = kLanes; x < 64; x *= 2) t += __shfl_xor(t, x, 64);
        if (lane < kLanes) cs[wave][h][r][lane * kCols + c] = t;
      }
  __syncthreads();
  if (wave != 0) return;
  const int row = lane / 8, unit = lane % 8;           // 8 columns of a row
  const int64_t at = col0 + unit * 8;
  const bool live = row < kM && row < a.end.rows && at < a.end.cols;
  float v[kHalves][8], residual[8];
#pragma unroll
  for (int h = 0; h < kHalves; ++h)
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const int i = unit * 8 + c, r = row < kM ? row : 0;
      v[h][c] = ((cs[0][h][r][i] + cs[1][h][r][i]) + cs[2][h][r][i]) + cs[3][h][r][i];
    }
  if (a.end.mode == kEndPartial) {
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
      store_partial(a.end, blockIdx.y, h, row < kM && row < a.end.rows, row, at, v[h]);
    return;
  }
  load_residual(kType, a.end, live, row, at, residual);
  finish(kType, a.end, live, row, at, v[0], v[kHalves - 1], residual);
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

int64_t rows_per_split(int64_t inner, int splits) { return ((inner + splits - 1) / splits + 31) / 32 * 32; }

}  // namespace

// About 4 blocks a CU, each over at least 128 inner indices.
int few_rows_splits(int64_t inner, int64_t cols, int halves, int cus) {
  const int64_t strips = (cols + kStrip - 1) / kStrip;
  int64_t s = 4 * (int64_t)cus / strips, most = (inner + 127) / 128;
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
