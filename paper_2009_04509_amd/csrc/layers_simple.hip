// The plain product kernel: any type, stride and size, fp32 arithmetic.
#include "internal.h"
#include "layers_end.h"

namespace pointid {
namespace {

constexpr int kTile = 32;        // rows and columns of a block
constexpr int kInner = 32;       // of the inner index at a time

// c[i][j] = sum over terms and k of left(i, k) right(j, k): a block of 256 threads
// computes 32 x 32 results (of each half), each thread 4 columns of one row, from tiles
// of 32 x 32 values held as fp32 in shared memory.
template <int kHalves>
__global__ void __launch_bounds__(256) simple_kernel(SimpleArgs a) {
  __shared__ float ls[kInner][kTile + 1];
  __shared__ float rs[kHalves][kInner][kTile + 4];
  __shared__ float cs[kHalves][kTile][kTile + 4];
  const int tid = threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.x * kTile, col0 = (int64_t)blockIdx.y * kTile;
  const int r = tid / 8, c = tid % 8 * 4;
  float acc[kHalves][4] = {};
  // the thread's place in a tile: consecutive threads along the operand's unit stride
  const int fast = tid % 32, slow = tid / 32;
  for (int t = 0; t < a.terms; ++t) {
    const Strided& L = a.left[t];
    const bool l_inner = L.sk == 1;
    for (int64_t k0 = 0; k0 < a.inner; k0 += kInner) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int i = l_inner ? slow + 8 * s : fast, k = l_inner ? fast : slow + 8 * s;
        ls[k][i] = row0 + i < a.end.rows && k0 + k < a.inner
                       ? load_any(L.p, (row0 + i) * L.si + (k0 + k) * L.sk, L.dtype) : 0.f;
      }
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        const Strided& R = a.right[t][h];
        const bool r_inner = R.sk == 1;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int j = r_inner ? slow + 8 * s : fast, k = r_inner ? fast : slow + 8 * s;
          rs[h][k][j] = col0 + j < a.end.cols && k0 + k < a.inner
                            ? load_any(R.p, (col0 + j) * R.si + (k0 + k) * R.sk, R.dtype) : 0.f;
        }
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kInner; ++k) {
        const float l = ls[k][r];
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[h][j] += l * rs[h][k][c + j];
      }
      __syncthreads();
    }
  }
#pragma unroll
  for (int h = 0; h < kHalves; ++h)
#pragma unroll
    for (int j = 0; j < 4; ++j) cs[h][r][c + j] = acc[h][j];
  __syncthreads();
  if (tid >= 128) return;
  float v[kHalves][8], residual[8];
  const int64_t row = row0 + tid / 4, col = col0 + tid % 4 * 8;
  const bool live = row < a.end.rows && col < a.end.cols;
  load_residual(a.end.dtype, a.end, live, row, col, residual);
#pragma unroll
  for (int h = 0; h < kHalves; ++h)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[h][j] = cs[h][tid / 4][tid % 4 * 8 + j];
  finish(a.end.dtype, a.end, live, row, col, v[0], v[kHalves - 1], residual);
}

}  // namespace

hipError_t launch_layers_simple(const SimpleArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.end.rows + kTile - 1) / kTile), (unsigned)((a.end.cols + kTile - 1) / kTile));
  return a.end.halves == 2 ? launch_kernel(simple_kernel<2>, grid, dim3(256), 0, stream, a)
                           : launch_kernel(simple_kernel<1>, grid, dim3(256), 0, stream, a);
}

}  // namespace pointid
