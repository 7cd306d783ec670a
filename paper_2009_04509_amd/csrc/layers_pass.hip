// Passes over one matrix: operands laid out for the product kernels, 8-bit checkpoints
// written and read, the gradient before an activation with its column sums.  All are
// bound by the bytes they move.
#include "internal.h"
#include "layers_end.h"

namespace pointid {
namespace {

// Pieces of 8 columns of a row, from piece `first` on, every `step`-th.
template <class F>
__device__ __forceinline__ void each_piece(int64_t rows, int64_t pieces, int64_t first, int64_t step, F&& f) {
  const int64_t total = rows * pieces;
  for (int64_t i = first; i < total; i += step) {
    const int64_t row = total <= UINT32_MAX ? (int64_t)((uint32_t)i / (uint32_t)pieces) : i / pieces;
    f(row, (i - row * pieces) * 8);
  }
}

// code 2^(e - 127), 8 columns a lane.  16384 x 8192 to bf16: 70 us, 5.8 TB/s read and written.
__global__ void __launch_bounds__(256) checkpoint_load_kernel(Packed8 src, int64_t rows, int64_t cols, int dtype,
                                                              void* out, int64_t ld) {
  each_piece(rows, (cols + 7) / 8, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256,
             [&](int64_t row, int64_t col) {
    float v[8];
    load_codes(src, row, col, cols, v);
    store_cols<8>(out, row * ld + col, dtype, cols - col, v);
  });
}

// Jobs' blocks from the launch's block `first_block` on, by the blocks up to `end_block`:
// each job takes those from its first to the next job's.
__device__ __forceinline__ void run_fill_block(const FillJobs& a, uint32_t first_block, uint32_t end_block) {
  const uint32_t at = blockIdx.x - first_block;
  int j = 0;
  while (j + 1 < a.count && at >= a.job[j + 1].first) ++j;
  const FillJob& job = a.job[j];
  const uint32_t block = at - job.first, blocks = (j + 1 < a.count ? a.job[j + 1].first : end_block - first_block) - job.first;
  each_piece(job.rows, job.ld / 8, (int64_t)block * 256 + threadIdx.x, (int64_t)blocks * 256,
             [&](int64_t row, int64_t col) {
    float v[8] = {};
    if (job.kind == FillJob::kCopy)
      load_cols<8>(job.src, row * job.ld_src + col, job.dtype, job.cols - col, v);
    else if (col < job.cols)
      load_codes(job.packed, row, col, job.cols, v);
    // fp16 values from 63488 on are kept as 65536, which the type would hold as an infinity: the
    // nearest that it holds is 65504
    if (job.kind == FillJob::kLoad && job.dtype == POINTID_FP16)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __builtin_fabsf(v[i]) == 65536.f ? __builtin_copysignf(65504.f, v[i]) : v[i];
    store_cols<8>(job.out, row * job.ld + col, job.dtype, 8, v);
  });
}
__global__ void __launch_bounds__(256) fill_kernel(FillJobs a) { run_fill_block(a, 0, gridDim.x); }
__global__ void __launch_bounds__(256) sums_kernel(SumsJobs a) {
  __shared__ float sums[256 / 32 * 33];
  sum_columns<256>(a, blockIdx.x, sums);
}

// A block of 32 values by 4 neighbouring lanes, which exchange its maximum (see save_codes); a
// lane has two such pieces in flight (one: 82 us for 77).  Bound by the bytes: bf16 16384 x
// 8192 74-77 us, 5.3-5.5 TB/s read and written.
template <int kType>
__global__ void __launch_bounds__(256) checkpoint_save_kernel(const char* src, int64_t ld, int64_t rows, int64_t cols,
                                                              Packed8 out) {
  constexpr int kSize = kType == POINTID_FP32 ? 4 : 2;
  const int64_t lanes = (cols + kBlock8 - 1) / kBlock8 * 4, total = rows * lanes;
  const int64_t step = (int64_t)gridDim.x * 256;
  // every lane of a wave takes the same number of turns, as the exchange needs all 4 of a block
  const int64_t last = (total + 63) / 64 * 64;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < last; i += 2 * step) {
    int64_t row[2], col[2];
    int n[2];
    Raw8<kType> raw[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t at = i + u * step;
      const bool here = at < total;
      row[u] = !here ? 0 : total <= UINT32_MAX ? (int64_t)((uint32_t)at / (uint32_t)lanes) : at / lanes;
      col[u] = here ? (at - row[u] * lanes) * 8 : 0;
      n[u] = here ? piece_cols(cols, col[u]) : 0;
      raw[u].load(src + (row[u] * ld + col[u]) * kSize, n[u]);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float v[8];
      raw[u].values(v);
      save_codes(out.codes + row[u] * cols + col[u], out.exponents + row[u] * (lanes / 4) + col[u] / kBlock8, n[u] > 0,
                 col[u] % kBlock8 == 0, n[u], v);
    }
  }
}

// How the activations of a gradient are kept.
enum { kKeptNot = 0, kKeptWhole = 1, kKeptPacked = 2 };

// 8 values of a gradient brought before the activation: g of dy (dh), z of z (g, u).
template <int kHalves>
__device__ __forceinline__ void through8(int act, const float (&g)[8], const float (&z)[kHalves][8],
                                         float (&d)[kHalves][8]) {
  static_for<5>([&](auto a) {                   // the choice outside of the loop
    if (act == a) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float value;
        if constexpr (kHalves == 2) {
          d[0][i] = through(a, z[0][i], g[i] * z[1][i], &value);
          d[1][i] = g[i] * value;
        } else {
          d[0][i] = through(a, z[0][i], g[i], &value);
        }
      }
    }
  });
}

// The largest of 256 threads' values.
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t (&waves)[4]) {
#pragma unroll
  for (int x = 1; x < 64; x *= 2) {
    const uint32_t other = (uint32_t)__shfl_xor((int)v, x, 64);
    v = other > v ? other : v;
  }
  if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) v = waves[w] > v ? waves[w] : v;
  return v;
}

// dz = dy act'(z) (dg, du) reaches past fp16's largest value, and below its smallest, where
// the products are in range: it is kept times a power of two, which this pass is for.  It
// computes what the gradient pass does and leaves the largest finite magnitude of each block
// (the gradient pass takes the largest of these, so that no word is shared and cleared).  In the
// trace a gated 8192 x 8192 takes 90 us (4.5 TB/s read), from 8 bits 78-87, 1693 x 2048 7; twice
// the blocks gained nothing.  A call of those sizes is 70-85 and 8 us longer by it.
template <int kHalves, bool kPacked>
__global__ void __launch_bounds__(256) grad_max_kernel(GradArgs a) {
  __shared__ uint32_t waves[4];
  uint32_t top = 0;
  each_piece(a.rows, (a.cols + 7) / 8, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256,
             [&](int64_t row, int64_t col) {
    const int n = piece_cols(a.cols, col);
    Raw8<POINTID_FP16> dy;
    dy.load(static_cast<const char*>(a.dy) + (row * a.ld_dy + col) * 2, n);
    float g[8], z[kHalves][8], d[kHalves][8];
    dy.values(g);
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      if constexpr (kPacked) {
        load_codes(a.z[h].packed, row, col, a.cols, z[h]);
      } else {
        Raw8<POINTID_FP16> w;
        w.load(static_cast<const char*>(a.z[h].matrix) + (row * a.z[h].ld + col) * 2, n);
        w.values(z[h]);
      }
    }
    through8<kHalves>(a.act, g, z, d);
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t b = finite_bits(d[h][i]);
        top = b > top ? b : top;
      }
  });
  top = block_max(top, waves);
  if (threadIdx.x == 0) a.maxima[blockIdx.x] = top;
}

// dz = dy act'(z), or of a gated layer dg = dh u act'(g) and du = dh act(g), in fp32 and
// rounded once to the type that the products read; the column sums before the rounding.
// Each block: 8 kTurns rows x 256 columns (the blocks past those take the fill's jobs, which
// need nothing of the gradient); 8 rows by 32 pieces of 8 columns at a time, two such turns'
// reads in flight before any is used (a read used at once: 163 us for a gated 8192 x 8192 in
// bf16).  Bound by the bytes: that one from 8 bits 120 us, 4.5 TB/s read and written; with x's
// 8192 x 4096 from 8 bits beside it 153, 4.3 TB/s.  A block's sums are added by the sums' pass
// in order, not by atomics, so that the bits do not depend on which block is first.
template <int kType, int kHalves, int kKept, int kTurns>
__global__ void __launch_bounds__(256) grad_kernel(GradArgs a, FillJobs fill) {
  __shared__ float sums[8][256 + 8];
  const uint32_t row_blocks = a.row_blocks, grad_blocks = row_blocks * a.strips;
  if (blockIdx.x >= grad_blocks) {
    run_fill_block(fill, grad_blocks, gridDim.x);
    return;
  }
  float scale = 1.f;
  if constexpr (kType == POINTID_FP16) {
    if (a.maxima) {
      __shared__ uint32_t waves[4];
      uint32_t top = 0;
      for (uint32_t i = threadIdx.x; i < a.maxima_count; i += 256) top = a.maxima[i] > top ? a.maxima[i] : top;
      top = block_max(top, waves);
      // top = f 2^e, f in [1/2, 1): to [2^14, 2^15)
      int p = top == 0 ? 0 : 15 - __builtin_amdgcn_frexp_expf(__uint_as_float(top));
      p = p < 126 ? p : 126;
      scale = __builtin_amdgcn_ldexpf(1.f, p);
      if (blockIdx.x == 0 && threadIdx.x == 0) *a.unscale = __builtin_amdgcn_ldexpf(1.f, -p);
    }
  }
  const uint32_t strip = blockIdx.x / row_blocks, row_block = blockIdx.x - strip * row_blocks;
  constexpr int kSize = kType == POINTID_FP32 ? 4 : 2;
  const int piece = threadIdx.x % 32, sub = threadIdx.x / 32;
  const int64_t col = (int64_t)strip * 256 + piece * 8;
  const int n = piece_cols(a.cols, col);
  const int64_t row0 = (int64_t)row_block * (8 * kTurns) + sub;
  // rows from row0 on, and where the lane's pieces of them stand
  const int left = (int)(a.rows - row0 < 8 * kTurns ? a.rows - row0 : 8 * kTurns);
  const int64_t blocks8 = (a.cols + kBlock8 - 1) / kBlock8;
  const char* dy_at = static_cast<const char*>(a.dy) + (row0 * a.ld_dy + col) * kSize;
  const char* z_at[kHalves];
  const uint8_t* x_at[kHalves];
#pragma unroll
  for (int h = 0; h < kHalves; ++h) {
    if constexpr (kKept == kKeptWhole) z_at[h] = static_cast<const char*>(a.z[h].matrix) + (row0 * a.z[h].ld + col) * kSize;
    if constexpr (kKept == kKeptPacked) {
      z_at[h] = reinterpret_cast<const char*>(a.z[h].packed.codes) + row0 * a.cols + col;
      x_at[h] = a.z[h].packed.exponents + row0 * blocks8 + col / kBlock8;
    }
  }
  float total[kHalves][8] = {};
  constexpr int kAhead = kTurns < 2 ? kTurns : 2;
  if (n > 0) {
#pragma unroll
    for (int s = 0; s < kTurns; s += kAhead) {
      Raw8<kType> dy[kAhead], zw[kAhead][kHalves];
      RawCodes zp[kAhead][kHalves];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int r = 8 * (s + u), here = r < left ? n : 0;
        dy[u].load(dy_at + r * a.ld_dy * kSize, here);
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
          if constexpr (kKept == kKeptWhole) zw[u][h].load(z_at[h] + r * a.z[h].ld * kSize, here);
          if constexpr (kKept == kKeptPacked)
            zp[u][h].load(reinterpret_cast<const uint8_t*>(z_at[h]) + r * a.cols, x_at[h] + r * blocks8, here);
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int r = 8 * (s + u);
        if (r >= left) continue;
        float d[kHalves][8], z[kHalves][8] = {}, g[8];
        dy[u].values(g);
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
          if constexpr (kKept == kKeptWhole) zw[u][h].values(z[h]);
          if constexpr (kKept == kKeptPacked) zp[u][h].values(z[h]);
        }
        // (what does not exist reads as 0 and stays 0: so does the padding)
        through8<kHalves>(a.act, g, z, d);
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
#pragma unroll
          for (int i = 0; i < 8; ++i) total[h][i] += d[h][i];
          if (a.parts == 0) continue;
          const int64_t at = (row0 + r) * a.ld + col;
          if constexpr (kType == POINTID_FP32) {
            store_cols<8>(a.out[h], at, kType, 8, d[h]);
          } else {
            if constexpr (kType == POINTID_FP16)
#pragma unroll
              for (int i = 0; i < 8; ++i) d[h][i] *= scale;
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack16(d[h][2 * i], d[h][2 * i + 1], kType);
            uint16_t* o = static_cast<uint16_t*>(a.out[h]) + at;
            *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
            if (a.parts < 2) continue;
            float rest[8];                               // none beside an infinity or NaN
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              rest[i] = d[h][i] - from16((uint16_t)(w[i / 2] >> (16 * (i % 2))), kType);
              if ((__float_as_uint(rest[i]) & 0x7FFFFFFFu) >= 0x7F800000u) rest[i] = 0.f;
            }
            store_cols<8>(o + a.plane, 0, kType, 8, rest);
          }
        }
      }
    }
  }
  if (!a.col_part) return;
#pragma unroll
  for (int h = 0; h < kHalves; ++h) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[sub][piece * 8 + i] = total[h][i];
    __syncthreads();
    const int64_t c = (int64_t)strip * 256 + threadIdx.x;
    float t = 0.f;
#pragma unroll
    for (int s = 0; s < 8; ++s) t += sums[s][threadIdx.x];
    if (c < a.cols) a.col_part[((int64_t)row_block * kHalves + h) * a.cols + c] = t;
    __syncthreads();
  }
}

template <int kType, int kTurns>
hipError_t launch_grad(const GradArgs& a, const FillJobs& fill, dim3 grid, hipStream_t stream) {
  auto go = [&](auto kernel) { return launch_kernel(kernel, grid, dim3(256), 0, stream, a, fill); };
  if (a.halves == 2)
    return a.z[0].matrix ? go(grad_kernel<kType, 2, kKeptWhole, kTurns>) : go(grad_kernel<kType, 2, kKeptPacked, kTurns>);
  if (a.z[0].matrix) return go(grad_kernel<kType, 1, kKeptWhole, kTurns>);
  return a.z[0].packed.codes ? go(grad_kernel<kType, 1, kKeptPacked, kTurns>) : go(grad_kernel<kType, 1, kKeptNot, kTurns>);
}

// The sums of a split product: part 0, 1, ... in order, and then the end that a product
// without splits has in its own kernel.  A launch's latency, 4 to 6 us, more than its bytes.
// Units of 8 columns of a row of partials.  kSub == 1: a lane adds a unit's parts in
// order.  kSub == 8, for many parts: 8 lanes of a unit take every eighth part each, and
// their sums are added in order.
template <int kType, int kHalves, int kSub>
__global__ void __launch_bounds__(256) join_kernel(End e, const float* part, int64_t part_ld, int splits) {
  constexpr int kUnits = 256 / kSub;
  __shared__ __align__(16) float sums[kSub > 1 ? kSub : 1][kHalves][kSub > 1 ? kUnits * 8 : 1];
  const int64_t units = part_ld / 8, total = e.rows * units;
  const int unit = threadIdx.x % kUnits, sub = threadIdx.x / kUnits;
  const int64_t i = (int64_t)blockIdx.x * kUnits + unit;
  const bool here = i < total;
  const int64_t row = here ? i / units : 0, col = here ? (i - row * units) * 8 : 0;
  const bool live = here && col < e.cols;
  float v[kHalves][8] = {}, bias[2][8];
  Residual<kType> residual;
  if (sub == 0) {
    load_bias(e.bias0, col, e.cols, bias[0]);
    load_bias(e.bias1, col, e.cols, bias[1]);
    residual.load(residual.at(e, row, col), e.residual && live ? piece_cols(e.cols, col) : 0);
  }
  if (here) {
#pragma unroll 4
    for (int s = sub; s < splits; s += kSub)
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        float f[8];
        __builtin_memcpy(f, part + (((int64_t)s * kHalves + h) * e.rows + row) * part_ld + col, 32);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[h][j] += f[j];
      }
  }
  if constexpr (kSub > 1) {
    static_assert(kUnits * 8 == 256, "a column of each half a lane");
#pragma unroll
    for (int h = 0; h < kHalves; ++h) __builtin_memcpy(&sums[sub][h][unit * 8], v[h], 32);
    __syncthreads();
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      float t = sums[0][h][threadIdx.x];
#pragma unroll
      for (int s = 1; s < kSub; ++s) t += sums[s][h][threadIdx.x];
      sums[0][h][threadIdx.x] = t;
    }
    __syncthreads();
    if (sub != 0) return;
#pragma unroll
    for (int h = 0; h < kHalves; ++h) __builtin_memcpy(v[h], &sums[0][h][unit * 8], 32);
  }
  Targets<kType, kHalves> to;
  to.init(e, row, col);
  finish<kType, kHalves>(e, to, live, col % kBlock8 == 0, piece_cols(e.cols, col), v[0], v[kHalves - 1], bias[0], bias[1],
                         residual, unscale_of<kType>(e));
}

__global__ void __launch_bounds__(256) zero_kernel(void* out, int64_t ld, int dtype, int64_t rows, int64_t cols) {
  const int64_t total = rows * cols, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += step)
    store_any(out, i / cols * ld + i % cols, 0.f, dtype);
}

// blocks for `items` lanes of work, at most 8 rounds of the card's 256 CUs of 8 blocks
unsigned pass_blocks(int64_t items) {
  const int64_t b = (items + 255) / 256;
  return (unsigned)(b < 16384 ? (b > 0 ? b : 1) : 16384);
}

}  // namespace

namespace {
// Sets the jobs' first blocks; their number.
uint32_t spread_fill(FillJobs* jobs) {
  uint32_t blocks = 0;
  for (int j = 0; j < jobs->count; ++j) {
    FillJob& job = jobs->job[j];
    job.first = blocks;
    blocks += pass_blocks(job.rows * (job.ld / 8));
  }
  return blocks;
}
}  // namespace

hipError_t launch_layers_fill(FillJobs jobs, hipStream_t stream) {
  const uint32_t blocks = spread_fill(&jobs);
  if (blocks == 0) return hipSuccess;
  return launch_kernel(fill_kernel, dim3(blocks), dim3(256), 0, stream, jobs);
}

hipError_t launch_layers_sums(const SumsJobs& jobs, hipStream_t stream) {
  return launch_kernel(sums_kernel, dim3(jobs.blocks()), dim3(256), 0, stream, jobs);
}

hipError_t launch_checkpoint_load(const Packed8& src, int64_t rows, int64_t cols, int dtype, void* out, int64_t ld,
                                  hipStream_t stream) {
  return launch_kernel(checkpoint_load_kernel, dim3(pass_blocks(rows * ((cols + 7) / 8))), dim3(256), 0, stream, src,
                       rows, cols, dtype, out, ld);
}

hipError_t launch_checkpoint_save(const void* src, int64_t ld, int dtype, int64_t rows, int64_t cols,
                                  const Packed8& out, hipStream_t stream) {
  const dim3 grid(pass_blocks((rows * ((cols + 31) / 32) * 4 + 1) / 2));
  auto go = [&](auto kernel) {
    return launch_kernel(kernel, grid, dim3(256), 0, stream, static_cast<const char*>(src), ld, rows, cols, out);
  };
  switch (dtype) {
    case POINTID_FP32: return go(checkpoint_save_kernel<POINTID_FP32>);
    case POINTID_BF16: return go(checkpoint_save_kernel<POINTID_BF16>);
  }
  return go(checkpoint_save_kernel<POINTID_FP16>);
}

uint32_t grad_max_blocks(int64_t rows, int64_t cols) {
  const int64_t blocks = (rows * ((cols + 7) / 8) + 255) / 256;
  return (uint32_t)(blocks < kMostMaxima ? blocks : kMostMaxima);
}

hipError_t launch_layers_grad_max(const GradArgs& a, hipStream_t stream) {
  if (a.dtype != POINTID_FP16 || !a.maxima || a.maxima_count != grad_max_blocks(a.rows, a.cols)) return hipErrorInvalidValue;
  for (int h = 0; h < a.halves; ++h)
    if (!a.z[h].any() || !a.z[h].matrix != !a.z[0].matrix) return hipErrorInvalidValue;
  auto go = [&](auto kernel) { return launch_kernel(kernel, dim3(a.maxima_count), dim3(256), 0, stream, a); };
  if (a.halves == 2) return a.z[0].matrix ? go(grad_max_kernel<2, false>) : go(grad_max_kernel<2, true>);
  return a.z[0].matrix ? go(grad_max_kernel<1, false>) : go(grad_max_kernel<1, true>);
}

int grad_rows(int64_t rows, int64_t cols, int cus) {
  return ((rows + 31) / 32) * ((cols + 255) / 256) < 2 * cus ? 8 : 32;
}

hipError_t launch_layers_grad(GradArgs a, int block_rows, FillJobs fill, hipStream_t stream) {
  const int64_t width = a.parts != 0 && a.ld > a.cols ? a.ld : a.cols;
  const int64_t row_blocks = (a.rows + block_rows - 1) / block_rows, strips = (width + 255) / 256;
  const int64_t blocks = row_blocks * strips + spread_fill(&fill);
  if (blocks > INT32_MAX / 256 * 2) return hipErrorInvalidValue;
  a.row_blocks = (uint32_t)row_blocks;
  a.strips = (uint32_t)strips;
  const dim3 grid((unsigned)blocks);
  // the halves are kept alike (the caller checks)
  if (a.halves == 2 && (!a.z[0].matrix != !a.z[1].matrix || !a.z[0].any() || !a.z[1].any())) return hipErrorInvalidValue;
  auto go = [&](auto type) {
    constexpr int kType = type;
    return block_rows == 8 ? launch_grad<kType, 1>(a, fill, grid, stream) : launch_grad<kType, 4>(a, fill, grid, stream);
  };
  switch (a.dtype) {
    case POINTID_FP32: return go(std::integral_constant<int, POINTID_FP32>{});
    case POINTID_BF16: return go(std::integral_constant<int, POINTID_BF16>{});
  }
  return go(std::integral_constant<int, POINTID_FP16>{});
}

hipError_t launch_layers_zero(void* out, int64_t ld, int dtype, int64_t rows, int64_t cols, hipStream_t stream) {
  return launch_kernel(zero_kernel, dim3(pass_blocks(rows * cols)), dim3(256), 0, stream, out, ld, dtype, rows, cols);
}

hipError_t launch_layers_join(const End& end, const float* part, int64_t part_ld, int splits, hipStream_t stream) {
  const int64_t units = end.rows * (part_ld / 8);
  const int sub = splits >= 8 ? 8 : 1;
  const int64_t blocks = (units + 256 / sub - 1) / (256 / sub);
  if (blocks > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  auto go = [&](auto kernel) { return launch_kernel(kernel, grid, dim3(256), 0, stream, end, part, part_ld, splits); };
  auto type = [&](auto t) {
    constexpr int kType = t;
    if (end.halves == 2) return sub == 8 ? go(join_kernel<kType, 2, 8>) : go(join_kernel<kType, 2, 1>);
    return sub == 8 ? go(join_kernel<kType, 1, 8>) : go(join_kernel<kType, 1, 1>);
  };
  switch (end.dtype) {
    case POINTID_FP32: return type(std::integral_constant<int, POINTID_FP32>{});
    case POINTID_BF16: return type(std::integral_constant<int, POINTID_BF16>{});
  }
  return type(std::integral_constant<int, POINTID_FP16>{});
}

}  // namespace pointid
