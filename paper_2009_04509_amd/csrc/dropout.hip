// Dropout: y = drop(x) + residual, one pass (see random.h for the mask).
//
// A lane takes pieces of 8 columns: one call of the generator, 16 bits an element, and one 16-byte
// load and store of 16-bit values.  Bound by the bytes: bf16 16384 x 8192 with a residual 131 us, 6.1
// TB/s read and written, the vector units busy 60 % of the time (20 of their 32 x 32 -> 64 bit
// products, at a quarter of the rate, for 8 elements).  Rows that end inside a piece are read and written
// value by value there: 60000 x 303 34 us, x 304 20.  16 bits and not 32 an element: half the
// products, for a p that is rounded to 2^-16.
#include "internal.h"
#include "layers_end.h"
#include "norm.h"
#include "passing.h"

namespace pointid {
namespace {

template <int kType>
__global__ void __launch_bounds__(256) dropout_kernel(DropoutArgs a) {
  constexpr int kSize = kType == POINTID_FP32 ? 4 : 2;
  const DropKey key(a.drop);
  const int64_t pieces = (a.cols + 7) / 8, total = a.rows * pieces;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = total <= UINT32_MAX ? (int64_t)((uint32_t)i / (uint32_t)pieces) : i / pieces;
    const int64_t col = (i - row * pieces) * 8;
    const int n = piece_cols(a.cols, col);
    Raw8<kType> x, r;
    Passing<kType>::load(&x, a.x + (row * a.ld_x + col) * kSize, n, a.passing);
    if (a.residual) Passing<kType>::load(&r, a.residual + (row * a.ld_residual + col) * kSize, n, a.passing);
    float v[8];
    x.values(v);
    drop8(a.drop, key, row, col, v);
    if (a.residual) {
      float f[8];
      r.values(f);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += f[j];
    }
    Passing<kType>::store(a.y + (row * a.ld_y + col) * kSize, n, v, a.passing);
  }
}

}  // namespace

hipError_t launch_dropout(DropoutArgs a, hipStream_t stream) {
  a.passing = passes_cache(a.dtype, a.rows, a.cols, a.residual ? 3 : 2);
  const int64_t blocks = (a.rows * ((a.cols + 7) / 8) + 255) / 256;
  const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384));
  switch (a.dtype) {
    case POINTID_FP32: return launch_kernel(dropout_kernel<POINTID_FP32>, grid, dim3(256), 0, stream, a);
    case POINTID_BF16: return launch_kernel(dropout_kernel<POINTID_BF16>, grid, dim3(256), 0, stream, a);
  }
  return launch_kernel(dropout_kernel<POINTID_FP16>, grid, dim3(256), 0, stream, a);
}

}  // namespace pointid
