// The joint of two residual blocks: the norm after a block, its gate, dropout and residual,
// and the norm before the next block, forward and backward.
#include "internal.h"
#include "layers_end.h"
#include "norm.h"

namespace pointid {
namespace {

// Sums of two values over a block's threads, in the same order every time.
template <int kThreads>
__device__ __forceinline__ float2 block_sum(float a, float b, float2 (&waves)[kThreads / 64]) {
#pragma unroll
  for (int x = 1; x < 64; x *= 2) {
    a += __shfl_xor(a, x, 64);
    b += __shfl_xor(b, x, 64);
  }
  __syncthreads();                             // the last call's sums have been read
  if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = make_float2(a, b);
  __syncthreads();
  float2 s = waves[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) {
    s.x += waves[w].x;
    s.y += waves[w].y;
  }
  return s;
}

template <int kType>
__device__ __forceinline__ void load_row(const Rows& m, int64_t row, int64_t col, int n, float (&v)[8]) {
  Raw8<kType> r;
  r.load(m.p + (row * m.ld + col) * (kType == POINTID_FP32 ? 4 : 2), n);
  r.values(v);
}
// 8 parameters of columns col on, n of them; `none` where there are none
__device__ __forceinline__ void load_param(const float* p, int64_t col, int n, float none, float (&v)[8]) {
  if (p) {
    load_cols<8>(p, col, POINTID_FP32, n, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = none;
}

struct Stats {
  float mean, r;
};
// v -> u = (v - mean) r, and u weight + bias
__device__ __forceinline__ void affine8(const NormOf& norm, const Stats& s, int64_t col, int n, float (&v)[8]) {
  float w[8], b[8];
  load_param(norm.weight, col, n, 1.f, w);
  load_param(norm.bias, col, n, 0.f, b);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (v[i] - s.mean) * s.r * w[i] + b[i];
}

// t of 8 columns
template <int kType>
__device__ __forceinline__ void total8(const NormArgs& a, const DropKey& key, const Stats& after, int64_t row,
                                       int64_t col, int n, float (&t)[8]) {
  load_row<kType>(a.x, row, col, n, t);
  if (!a.o.p) return;
  float v[8], g[8];
  load_row<kType>(a.o, row, col, n, v);
  if (a.after.kind) affine8(a.after, after, col, n, v);
  if (a.drop.threshold) drop8(a.drop, key, row, col, v);
  load_param(a.gate, col, n, 1.f, g);
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = a.scale * t[i] + g[i] * v[i];
}

// The mean (layer) and one over the deviation of a row whose 8 values from a column on `at` gives.
// The squares are of the values less the mean, in a pass of their own.
template <class At>
__device__ __forceinline__ Stats stats_of(const NormOf& norm, int64_t cols, float2 (&waves)[4], At&& at) {
  Stats s = {0.f, 1.f};
  float f[8];
  if (norm.kind == POINTID_NORM_LAYER) {
    float sum = 0.f;
    for (int64_t col = threadIdx.x * 8; col < cols; col += 256 * 8) {
      at(col, piece_cols(cols, col), f);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += col + i < cols ? f[i] : 0.f;
    }
    s.mean = block_sum<256>(sum, 0.f, waves).x / (float)cols;
  }
  float sum = 0.f;
  for (int64_t col = threadIdx.x * 8; col < cols; col += 256 * 8) {
    at(col, piece_cols(cols, col), f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float d = f[i] - s.mean;
      sum += col + i < cols ? d * d : 0.f;
    }
  }
  s.r = 1.f / sqrtf(block_sum<256>(sum, 0.f, waves).x / (float)cols + norm.eps);
  return s;
}

template <int kType>
__global__ void __launch_bounds__(256) norm_kernel(NormArgs a) {
  __shared__ float2 waves[4];
  const DropKey key(a.drop);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    Stats after = {0.f, 1.f}, before = {0.f, 1.f};
    if (a.o.p && a.after.kind)
      after = stats_of(a.after, a.cols, waves,
                       [&](int64_t col, int n, float (&v)[8]) { load_row<kType>(a.o, row, col, n, v); });
    if (a.before.kind)
      before = stats_of(a.before, a.cols, waves,
                        [&](int64_t col, int n, float (&v)[8]) { total8<kType>(a, key, after, row, col, n, v); });
    for (int64_t col = threadIdx.x * 8; col < a.cols; col += 256 * 8) {
      const int n = piece_cols(a.cols, col);
      float t[8];
      total8<kType>(a, key, after, row, col, n, t);
      if (a.t.p) store_cols<8>(a.t.p, row * a.t.ld + col, kType, n, t);
      if (!a.h.p) continue;
      affine8(a.before, before, col, n, t);
      store_cols<8>(a.h.p, row * a.h.ld + col, kType, n, t);
    }
    if (a.stats && threadIdx.x == 0)
      reinterpret_cast<float4*>(a.stats)[row] = make_float4(after.mean, after.r, before.mean, before.r);
  }
}

// ---- backward.  With u_b = (t - mean) r of the norm before the next block and u_a of the one
// after this one, v = u_a w_a + b_a (without that norm: o) and k the dropout's factor:
//   e = dh w_b         d = dt + r_b (e - mean(e u_b) u_b - [layer] mean(e))
//   f = d k g w_a      do = r_a (f - mean(f u_a) u_a - [layer] mean(f))      dx = scale d
//   dw_b = sum dh u_b   db_b = sum dh   dw_a = sum d k g u_a   db_a = sum d k g   dg = sum d k v

struct Back8 {
  float d[8];                  // the gradient of t
  float q[8];                  // d k g
  float u_a[8];                // without a norm after the block: o
};
// dh, t -> e and u_b of 8 columns; e u_b and e are 0 past n
template <int kType>
__device__ __forceinline__ void before8(const NormBackArgs& a, const float4& st, int64_t row, int64_t col, int n,
                                        float (&dh)[8], float (&u)[8]) {
  load_row<kType>(a.dh, row, col, n, dh);
  load_row<kType>(a.t, row, col, n, u);
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = (u[i] - st.z) * st.w;
}
template <int kType>
__device__ __forceinline__ void back8(const NormBackArgs& a, const DropKey& key, const float4& st, float mean_e,
                                      float mean_eu, int64_t row, int64_t col, int n, Back8* b, float (&dh)[8],
                                      float (&u_b)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) b->d[i] = 0.f;
  if (a.dt.p) load_row<kType>(a.dt, row, col, n, b->d);
  if (a.before.kind) {
    float w[8];
    before8<kType>(a, st, row, col, n, dh, u_b);
    load_param(a.before.weight, col, n, 1.f, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) b->d[i] += st.w * (dh[i] * w[i] - mean_eu * u_b[i] - mean_e);
  }
  if (!a.o.p && !a.dout.p) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) b->q[i] = b->d[i];
  if (a.drop.threshold) drop8(a.drop, key, row, col, b->q);
  if (a.o.p) {
    load_row<kType>(a.o, row, col, n, b->u_a);
    if (a.after.kind)
#pragma unroll
      for (int i = 0; i < 8; ++i) b->u_a[i] = (b->u_a[i] - st.x) * st.y;
  }
}

// The means over each row that its gradients take: of e and e u_b, then of f and f u_a.
template <int kType>
__global__ void __launch_bounds__(256) norm_means_kernel(NormBackArgs a) {
  __shared__ float2 waves[4];
  const DropKey key(a.drop);
  const float inv = 1.f / (float)a.cols;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float4 st = reinterpret_cast<const float4*>(a.stats)[row];
    float4 m = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.before.kind) {
      float se = 0.f, seu = 0.f;
      for (int64_t col = threadIdx.x * 8; col < a.cols; col += 256 * 8) {
        const int n = piece_cols(a.cols, col);
        float dh[8], u[8], w[8];
        before8<kType>(a, st, row, col, n, dh, u);
        load_param(a.before.weight, col, n, 1.f, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (i >= n) continue;
          se += dh[i] * w[i];
          seu += dh[i] * w[i] * u[i];
        }
      }
      const float2 s = block_sum<256>(se, seu, waves);
      m.x = a.before.kind == POINTID_NORM_LAYER ? s.x * inv : 0.f;
      m.y = s.y * inv;
    }
    if (a.after.kind && a.dout.p) {
      float sf = 0.f, sfu = 0.f;
      for (int64_t col = threadIdx.x * 8; col < a.cols; col += 256 * 8) {
        const int n = piece_cols(a.cols, col);
        Back8 b;
        float dh[8], u[8], w[8], g[8];
        back8<kType>(a, key, st, m.x, m.y, row, col, n, &b, dh, u);
        load_param(a.after.weight, col, n, 1.f, w);
        load_param(a.gate, col, n, 1.f, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (i >= n) continue;
          const float f = b.q[i] * g[i] * w[i];
          sf += f;
          sfu += f * b.u_a[i];
        }
      }
      const float2 s = block_sum<256>(sf, sfu, waves);
      m.z = a.after.kind == POINTID_NORM_LAYER ? s.x * inv : 0.f;
      m.w = s.y * inv;
    }
    if (threadIdx.x == 0) reinterpret_cast<float4*>(a.means)[row] = m;
  }
}

// 8 rows x 256 columns at a time, by the blocks of rows that plan_norm_back gives.
template <int kType>
__global__ void __launch_bounds__(256) norm_back_kernel(NormBackArgs a) {
  __shared__ float sums[8][256 + 8];
  const DropKey key(a.drop);
  const int piece = threadIdx.x % 32, sub = threadIdx.x / 32;
  const int64_t col = (int64_t)blockIdx.x * 256 + piece * 8;
  const int n = piece_cols(a.cols, col);
  float total[kNormSums][8] = {};
  if (n > 0) {
    float w[8], bias[8], g[8];
    load_param(a.after.weight, col, n, 1.f, w);
    load_param(a.after.bias, col, n, 0.f, bias);
    load_param(a.gate, col, n, 1.f, g);
    for (int64_t row = (int64_t)blockIdx.y * 8 + sub; row < a.rows; row += (int64_t)gridDim.y * 8) {
      const float4 st = a.stats ? reinterpret_cast<const float4*>(a.stats)[row] : make_float4(0.f, 1.f, 0.f, 1.f);
      const float4 m = a.means ? reinterpret_cast<const float4*>(a.means)[row] : make_float4(0.f, 0.f, 0.f, 0.f);
      Back8 b;
      float dh[8] = {}, u_b[8] = {}, v[8];
      back8<kType>(a, key, st, m.x, m.y, row, col, n, &b, dh, u_b);
      if (a.dx.p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = a.scale * b.d[i];
        store_cols<8>(a.dx.p, row * a.dx.ld + col, kType, n, v);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        total[0][i] += dh[i] * u_b[i];
        total[1][i] += dh[i];
      }
      if (!a.o.p && !a.dout.p) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float q = b.q[i] * g[i];
        if (a.o.p) {
          total[4][i] += b.q[i] * (a.after.kind ? b.u_a[i] * w[i] + bias[i] : b.u_a[i]);
          total[2][i] += q * b.u_a[i];
        }
        total[3][i] += q;
        v[i] = a.after.kind ? st.y * (q * w[i] - m.w * b.u_a[i] - m.z) : q;
      }
      if (a.dout.p) store_cols<8>(a.dout.p, row * a.dout.ld + col, kType, n, v);
    }
  }
  int wanted = 0, at = 0;
  for (int s = 0; s < kNormSums; ++s) wanted += a.out[s] != nullptr;
#pragma unroll
  for (int s = 0; s < kNormSums; ++s) {
    if (!a.out[s]) continue;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[sub][piece * 8 + i] = total[s][i];
    __syncthreads();
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    float t = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) t += sums[r][threadIdx.x];
    if (c < a.cols) a.part[((int64_t)blockIdx.y * wanted + at) * a.cols + c] = t;
    ++at;
  }
}

// The sums of the blocks' sums: 32 columns of one parameter a block, 8 of the partial rows
// at a time, added in order.
__global__ void __launch_bounds__(256) norm_sums_kernel(NormBackArgs a) {
  __shared__ float sums[8][33];
  int wanted = 0, which = 0, at = 0;
  for (int s = 0; s < kNormSums; ++s) {
    if (!a.out[s]) continue;
    if (wanted == (int)blockIdx.y) which = s, at = wanted;
    ++wanted;
  }
  const int c = threadIdx.x % 32, sub = threadIdx.x / 32;
  const int64_t col = (int64_t)blockIdx.x * 32 + c;
  float t = 0.f;
  if (col < a.cols)
#pragma unroll 4
    for (int b = sub; b < a.blocks; b += 8) t += a.part[((int64_t)b * wanted + at) * a.cols + col];
  sums[sub][c] = t;
  __syncthreads();
  if (sub != 0 || col >= a.cols) return;
  t = 0.f;
#pragma unroll
  for (int s = 0; s < 8; ++s) t += sums[s][c];
  a.out[which][col] = t;
}

unsigned row_blocks(int64_t rows) { return (unsigned)(rows < 65536 ? rows : 65536); }

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
  const dim3 grid(row_blocks(a.rows));
  switch (a.dtype) {
    case POINTID_FP32: return launch_kernel(norm_kernel<POINTID_FP32>, grid, dim3(256), 0, stream, a);
    case POINTID_BF16: return launch_kernel(norm_kernel<POINTID_BF16>, grid, dim3(256), 0, stream, a);
  }
  return launch_kernel(norm_kernel<POINTID_FP16>, grid, dim3(256), 0, stream, a);
}

NormBackPlan plan_norm_back(const NormBackArgs& a, int cus) {
  const int64_t strips = (a.cols + 255) / 256, most = (a.rows + 31) / 32, want = (8 * cus + strips - 1) / strips;
  NormBackPlan p;
  p.blocks = (int32_t)(most < want ? most : want);
  p.means = a.before.kind || (a.after.kind && a.dout.p);
  return p;
}

hipError_t launch_norm_means(const NormBackArgs& a, hipStream_t stream) {
  const dim3 grid(row_blocks(a.rows));
  switch (a.dtype) {
    case POINTID_FP32: return launch_kernel(norm_means_kernel<POINTID_FP32>, grid, dim3(256), 0, stream, a);
    case POINTID_BF16: return launch_kernel(norm_means_kernel<POINTID_BF16>, grid, dim3(256), 0, stream, a);
  }
  return launch_kernel(norm_means_kernel<POINTID_FP16>, grid, dim3(256), 0, stream, a);
}

hipError_t launch_norm_back(const NormBackArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.cols + 255) / 256), (unsigned)a.blocks);
  switch (a.dtype) {
    case POINTID_FP32: return launch_kernel(norm_back_kernel<POINTID_FP32>, grid, dim3(256), 0, stream, a);
    case POINTID_BF16: return launch_kernel(norm_back_kernel<POINTID_BF16>, grid, dim3(256), 0, stream, a);
  }
  return launch_kernel(norm_back_kernel<POINTID_FP16>, grid, dim3(256), 0, stream, a);
}

hipError_t launch_norm_sums(const NormBackArgs& a, hipStream_t stream) {
  int wanted = 0;
  for (int s = 0; s < kNormSums; ++s) wanted += a.out[s] != nullptr;
  return launch_kernel(norm_sums_kernel, dim3((unsigned)((a.cols + 31) / 32), (unsigned)wanted), dim3(256), 0, stream,
                       a);
}

}  // namespace pointid
