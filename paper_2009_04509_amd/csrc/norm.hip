// The joint of two residual blocks: the norm after a block, its gate, dropout and residual,
// and the norm before the next block, forward and backward:
//   v = after(o)   t = scale x + gate * drop(v)   h = before(t)
// All are bound by the bytes of their matrices.  A row is held in registers, 8 columns (16 bytes of
// 16-bit values) a thread, from one load to the last store, where a block can hold it: forward up to
// 16384 columns, backward up to 8192; wider rows are read again for each sum.  The squares of a layer
// norm are of what the mean leaves, so that a mean far from zero costs no more than its own rounding.
#include "internal.h"
#include "layers_end.h"
#include "norm.h"
#include "passing.h"
#include "wave.h"

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

// A layer norm's statistics.  `about`: the mean but for the roundings of its sum; rest and squares: the
// means of what is left of the values and of its squares.  What is left, small as it is, holds the
// sum's roundings: with it the mean is rounded once, and a row of one value has that as its mean.
__device__ __forceinline__ Stats layer_stats(const NormOf& norm, float about, float rest, float squares) {
  const float spread = squares - rest * rest;
  // (squares past fp32's range stay so)
  if (squares < __builtin_inff()) squares = fmaxf(spread, 0.f);
  return {about + rest, 1.f / sqrtf(squares + norm.eps)};
}

// The mean (layer) and one over the deviation of a row whose 8 values from a column on `at` gives.
// The squares are of the values less the mean, in a pass of their own.
template <class At>
__device__ __forceinline__ Stats stats_of(const NormOf& norm, int64_t cols, float2 (&waves)[4], At&& at) {
  float f[8], about = 0.f;
  if (norm.kind == POINTID_NORM_LAYER) {
    float sum = 0.f;
    for (int64_t col = threadIdx.x * 8; col < cols; col += 256 * 8) {
      at(col, piece_cols(cols, col), f);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += col + i < cols ? f[i] : 0.f;
    }
    about = block_sum<256>(sum, 0.f, waves).x / (float)cols;
  }
  float sum = 0.f, squares = 0.f;
  for (int64_t col = threadIdx.x * 8; col < cols; col += 256 * 8) {
    at(col, piece_cols(cols, col), f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float d = col + i < cols ? f[i] - about : 0.f;
      sum += d;
      squares += d * d;
    }
  }
  const float2 s = block_sum<256>(sum, squares, waves);
  const float n = (float)cols;
  if (norm.kind == POINTID_NORM_LAYER) return layer_stats(norm, about, s.x / n, s.y / n);
  return {0.f, 1.f / sqrtf(s.y / n + norm.eps)};
}

// Rows of more than 16384 columns: a block a row, which is read once for each sum and once more.  bf16,
// both norms and a gate, 4096 x 16400 210 us and 4096 x 32768 438 (held, 4096 x 16384 126).
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

// ---- rows held in registers: a block's threads are groups of `lanes`, each group with a row at
// a time and each thread with 8 columns of it

constexpr int kMostWaves = 16;

// Sums over a group: 16 lanes (kSmall), or whole waves, which exchange theirs with one barrier of
// the block a call: the buffers take turns, so that a call's are not written again before the
// next call's barrier.
template <bool kSmall>
struct RowSum {
  float2 (*waves)[kMostWaves];
  int first, count;            // the group's waves
  int turn = 0;
  __device__ __forceinline__ RowSum(float2 (*w)[kMostWaves], int lanes)
      : waves(w), first((int)threadIdx.x / lanes * (lanes / 64)), count(lanes / 64) {}
  __device__ __forceinline__ float2 operator()(float a, float b) {
    if constexpr (kSmall) return make_float2(lanes_sum<16>(a), lanes_sum<16>(b));
    a = lanes_sum<64>(a);
    b = lanes_sum<64>(b);
    if (count == 1) return make_float2(a, b);
    const int lane = threadIdx.x % 64;
    if (lane == 0) waves[turn][threadIdx.x / 64] = make_float2(a, b);
    __syncthreads();
    const float2 s = lane % 16 < count ? waves[turn][first + lane % 16] : make_float2(0.f, 0.f);
    turn ^= 1;
    return make_float2(lanes_sum<16>(s.x), lanes_sum<16>(s.y));
  }
  __device__ __forceinline__ float operator()(float a) {
    if constexpr (kSmall) return lanes_sum<16>(a);
    return (*this)(a, 0.f).x;
  }
};

// A value that a wave's threads have alike, in a register of the wave's.
__device__ __forceinline__ float of_wave(float v) {
  return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}
// A thread's group; known to be the same for a wave's threads where it is.
template <bool kSmall>
__device__ __forceinline__ int group_of(int lanes) {
  if constexpr (kSmall) return threadIdx.x / 16;
  return __builtin_amdgcn_readfirstlane((int)threadIdx.x / lanes);
}

// How rows end: with a whole piece of 8 columns; with a ragged one, which is read as the row's last 8
// columns, a load like the others, and moved into place when it is used; or before the eighth column.
// (Read value by value, each load would be waited for with all that is on its way beside it: bf16 5280 x
// 4287, both norms and a gate, 52 us for 73, the gradients 82 for 161; 5280 x 4288 takes 40 and 61.)
enum { kWhole = 0, kRagged = 1, kTiny = 2 };

// A thread's columns of a row: kPieces pieces of 8, a row's threads apart.
template <int kEnd, int kPieces>
struct Columns {
  int col[kPieces], n[kPieces];  // first column, and how many exist
  int from[kPieces];             // the column from which on 8 are read
  bool any_end[kPieces];         // a thread of the wave has less than a whole piece
  __device__ __forceinline__ Columns(int64_t cols, int lane, int lanes) {
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      col[p] = (p * lanes + lane) * 8;
      n[p] = piece_cols(cols, col[p]);
      from[p] = kEnd == kRagged && n[p] < 8 ? (int)cols - 8 : col[p];
      any_end[p] = __any(n[p] < 8);
    }
  }
};

// A thread's columns of one matrix, row after row.
template <int kType, int kEnd, int kPieces>
struct Stream {
  static constexpr int64_t kSize = kType == POINTID_FP32 ? 4 : 2;
  char* p;                     // the next row's first column, nullptr without a matrix
  int64_t step;                // bytes to the group's row after it
  bool passing;
  Raw8<kType> raw[kPieces];
  __device__ __forceinline__ Stream(const Rows& m, int64_t row, int64_t rows_on, bool passing_)
      : p(m.p ? m.p + row * m.ld * kSize : nullptr), step(rows_on * m.ld * kSize), passing(passing_) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) raw[i].load(nullptr, 0);
  }
  // the next row, if there is one (`here`), on its way; zeros if not
  __device__ __forceinline__ void load(const Columns<kEnd, kPieces>& c, bool here) {
    if (!p) return;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      if (!here)
        raw[i].load(nullptr, 0);
      else if constexpr (kEnd == kTiny)
        raw[i].load(p + c.col[i] * kSize, c.n[i]);
      else if (kEnd == kRagged || c.n[i] > 0)
        Passing<kType>::load(&raw[i], p + c.from[i] * kSize, 8, passing);
    }
    p += step;
  }
  // the values of a piece, 0 where there is no column
  __device__ __forceinline__ void values(int i, const Columns<kEnd, kPieces>& c, float (&v)[8]) const {
    raw[i].values(v);
    if constexpr (kEnd == kRagged)
      if (c.any_end[i]) {                        // a branch of the whole wave
        const int move = c.col[i] - c.from[i];
        move_down<4>(move, v);
        move_down<2>(move, v);
        move_down<1>(move, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < c.n[i] ? v[k] : 0.f;
      }
  }
  // kBy to the left, in bits: a choice between two places would be one between addresses, in memory
  template <int kBy>
  static __device__ __forceinline__ void move_down(int move, float (&v)[8]) {
    const int mask = (move & kBy) != 0 ? -1 : 0;
#pragma unroll
    for (int k = 0; k < 8 - kBy; ++k) {
      const int here = __float_as_int(v[k]), there = __float_as_int(v[k + kBy]);
      v[k] = __int_as_float(here ^ ((here ^ there) & mask));
    }
  }
  // one piece of the row, and on to the next (a matrix that is not there stays so)
  __device__ __forceinline__ void store(int col, int n, bool here, const float (&v)[8]) const {
    if (p && here && n > 0) Passing<kType>::store(p + col * kSize, kEnd == kWhole ? 8 : n, v, passing);
  }
  __device__ __forceinline__ void next() {
    if (p) p += step;
  }
};

// A parameter's 8 columns of a thread from shared memory, where it stands as [2][lanes] pieces
// of 4 (reads of a wave without bank conflicts).
__device__ __forceinline__ void share_param(const float* p, float none, float4* to, int lanes, int lane, int col, int n) {
  float v[8];
  load_param(p, col, n, none, v);
  to[lane] = make_float4(v[0], v[1], v[2], v[3]);
  to[lanes + lane] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void shared_param(const float4* from, int lanes, int lane, float (&v)[8]) {
  const float4 a = from[lane], b = from[lanes + lane];
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
  v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}

// 0 past the n columns of a piece, in the waves that have such.
__device__ __forceinline__ void zero_past(bool any_end, int n, float (&v)[8]) {
  if (any_end)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] : 0.f;
}

// A quotient sum / n, rounded once, from 1 / n: not made part of what it is subtracted from.
__device__ __forceinline__ float quotient(float sum, float n, float inv) {
#pragma clang fp contract(off)
  const float q = sum * inv;
  return q + __builtin_fmaf(-q, n, sum) * inv;
}

// The mean (layer) and 1 / deviation of a row, whose values are 0 past its columns.  The mean of one
// value in every column is that value, or u is not 0 (with the sum times 1 / n, a bf16 row of 1000s had u
// -0.02 at 5280 columns).  Of 16-bit values their sum's quotient holds it, as the sum is exact; of fp32
// values what is left of them has to be summed too, which is time that 16-bit rows have not got (bf16
// 16384 x 4096, two layer norms 124 us for 119, 5280 x 4288 71 for 67; fp32 8192 x 4096 109 for 109).
template <int kType, int kEnd, int kPieces, class S>
__device__ __forceinline__ Stats held_stats(const NormOf& norm, float cols, float inv, const Columns<kEnd, kPieces>& c,
                                            S& row_sum, const float (&v)[kPieces][8]) {
  float about = 0.f, sum = 0.f, squares = 0.f;
  if (norm.kind == POINTID_NORM_LAYER) {
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += v[p][i];
    about = quotient(row_sum(sum), cols, inv);
    sum = 0.f;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      float d[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = v[p][i] - about;
      zero_past(c.any_end[p], c.n[p], d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (kType == POINTID_FP32) sum += d[i];
        squares += d[i] * d[i];
      }
    }
    if constexpr (kType == POINTID_FP32) {
      const float2 rest = row_sum(sum, squares);
      return layer_stats(norm, about, rest.x * inv, rest.y * inv);
    }
  } else {
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) squares += v[p][i] * v[p][i];
  }
  return {about, 1.f / sqrtf(row_sum(squares) * inv + norm.eps)};
}

extern __shared__ float4 shared_floats[];

// The parameters, in the order in which they stand in shared memory, in blocks of 2 lanes pieces.
enum { kAfterWeight = 0, kGate = 1, kBeforeWeight = 2, kAfterBias = 3, kBeforeBias = 4 };
template <int kParam>
using Which = std::integral_constant<int, kParam>;
template <class Args>
__device__ __forceinline__ const float* param_of(const Args& a, int i) {
  return i == kAfterWeight ? a.after.weight : i == kGate ? a.gate : i == kBeforeWeight ? a.before.weight
         : i == kAfterBias ? a.after.bias : a.before.bias;
}

// kShared: that many of the parameters wait in shared memory, for blocks of many rows.  What is not
// given counts as ones and zeros.
// bf16 16384 x 4096 with both norms and a gate (537 MB): 102 us, 5.3 TB/s, the vector units busy
// 55 %.  256 threads of two pieces with the parameters in registers took 147 (173 registers: two
// waves a SIMD), blocks of 1024 threads in two groups 138, parameters from memory 121.
template <int kType, bool kSmall, int kEnd, bool kBiases, int kShared, int kPieces>
__global__ void __launch_bounds__(1024) norm_rows_kernel(NormArgs a) {
  static_assert(kShared == 0 || kPieces == 1, "parameters of one piece a thread");
  __shared__ float2 waves[2][kMostWaves];
  const int lanes = kSmall ? 16 : a.lanes, groups = blockDim.x / lanes, group = group_of<kSmall>(lanes);
  const int lane = threadIdx.x - group * lanes;
  const Columns<kEnd, kPieces> c(a.cols, lane, lanes);
  const int (&col)[kPieces] = c.col, (&n)[kPieces] = c.n;
  RowSum<kSmall> row_sum(waves, lanes);
  const DropKey key(a.drop);
  const float cols = of_wave((float)a.cols), inv = of_wave(1.f / (float)a.cols);
  const int64_t step = (int64_t)gridDim.x * groups;
  int64_t row = (int64_t)blockIdx.x * groups + group;
  Stream<kType, kEnd, kPieces> x(a.x, row, step, a.passing), o(a.o, row, step, a.passing);
  Stream<kType, kEnd, kPieces> t(a.t, row, step, a.passing), h(a.h, row, step, a.passing);
  o.load(c, row < a.rows);
  x.load(c, row < a.rows);
  if constexpr (kShared > 0) {
#pragma unroll
    for (int i = 0; i < kShared; ++i)
      if (i % groups == group)
        share_param(param_of(a, i), i < 3 ? 1.f : 0.f, shared_floats + i * 2 * lanes, lanes, lane, col[0], n[0]);
    __syncthreads();
  }
  auto param = [&](auto which, int p, float (&v)[8]) {
    constexpr int i = decltype(which)::value;
    if constexpr (i < kShared)
      shared_param(shared_floats + i * 2 * lanes, lanes, lane, v);
    else
      load_param(param_of(a, i), col[p], n[p], i < 3 ? 1.f : 0.f, v);
  };
  // (v - mean) r weight + bias
  auto affine = [&](float (&v)[8], const Stats& s, auto weight, auto bias, int p) {
    float w[8];
    param(weight, p, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (v[i] - s.mean) * s.r * w[i];
    if constexpr (kBiases) {
      param(bias, p, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += w[i];
    }
  };
  // every group takes the same number of turns, as the sums need the whole block
  for (int64_t first = (int64_t)blockIdx.x * groups; first < a.rows; first += step, row += step) {
    const bool here = row < a.rows, more = row + step < a.rows;
    float v[kPieces][8], s[kPieces][8];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      o.values(p, c, v[p]);
      x.values(p, c, s[p]);
    }
    // the next row is on its way while this one is worked on
    o.load(c, more);
    x.load(c, more);
    Stats after = {0.f, 1.f}, before = {0.f, 1.f};
    if (a.o.p) {
      if (a.after.kind) {
        after = held_stats<kType>(a.after, cols, inv, c, row_sum, v);
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
          affine(v[p], after, Which<kAfterWeight>{}, Which<kAfterBias>{}, p);
          zero_past(c.any_end[p], n[p], v[p]);
        }
      }
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        if (a.drop.threshold) drop8(a.drop, key, row, col[p], v[p]);
        if (a.gate) {
          float w[8];
          param(Which<kGate>{}, p, w);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[p][i] *= w[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) s[p][i] = a.scale * s[p][i] + v[p][i];
        t.store(col[p], n[p], here, s[p]);
      }
      t.next();
    }
    if (a.h.p) {
      before = held_stats<kType>(a.before, cols, inv, c, row_sum, s);
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        affine(s[p], before, Which<kBeforeWeight>{}, Which<kBeforeBias>{}, p);
        h.store(col[p], n[p], here, s[p]);
      }
      h.next();
    }
    if (a.stats && lane == 0 && here)
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
#pragma unroll
  for (int i = 0; i < 8; ++i) b->u_a[i] = 0.f;
  if (a.o.p) load_row<kType>(a.o, row, col, n, b->u_a);
  // (o's own infinities do not reach the gate's gradient where they are dropped; a norm's whole row
  // has them)
  if (a.drop.threshold) {
    if (a.after.kind)
      drop8(a.drop, key, row, col, b->q);
    else
      drop8(a.drop, key, row, col, b->q, &b->u_a);
  }
  if (a.after.kind)
#pragma unroll
    for (int i = 0; i < 8; ++i) b->u_a[i] = (b->u_a[i] - st.x) * st.y;
}

// Rows of more than 8192 columns take two passes: the means over each row that its gradients take,
// of e and e u_b, then of f and f u_a (the row read again for these), and what is made of them, with
// the column sums, in strips of 256 columns.  bf16 4096 x 16384 (805 MB) 330 us; held rows of half
// the width 166.
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

// Both passes and the column sums with the rows held in registers; each block takes every
// gridDim-th set of rows, one of each of its groups, and leaves its sums (the only block: the sums):
// one block a CU, so that there are few sums to add.  A norm that there is not has the mean 0, the
// deviation 1, and means of its gradient that count as 0.
// bf16 16384 x 4096 with dropout (805 MB): 139 us, 5.8 TB/s, the vector units busy 65 %, and 4.8 for the
// sums.  A branch for each part that a call may lack, and its parameters in registers (167: three waves
// a SIMD, one block of 512 threads), took 277; both in shared memory and the branches 230.  fp16 1693
// x 2304, layer norms (47 MB): 21 us, 3.3 rows for each of 512 groups, of which the first waits for
// memory.
template <int kType, bool kSmall, int kEnd, bool kBiases, int kMost>
__global__ void __launch_bounds__(kMost) norm_back_rows_kernel(NormBackArgs a) {
  __shared__ float2 waves[2][kMostWaves];
  const int lanes = kSmall ? 16 : a.lanes, groups = blockDim.x / lanes, group = group_of<kSmall>(lanes);
  const int lane = threadIdx.x - group * lanes, col = lane * 8, n = piece_cols(a.cols, col);
  const Columns<kEnd, 1> c(a.cols, lane, lanes);
  RowSum<kSmall> row_sum(waves, lanes);
  const DropKey key(a.drop);
  const float inv = 1.f / (float)a.cols;
  const int64_t step = (int64_t)gridDim.x * groups;
  int64_t row = (int64_t)blockIdx.x * groups + group;
  Stream<kType, kEnd, 1> dh(a.dh, row, step, a.passing), t(a.t, row, step, a.passing);
  Stream<kType, kEnd, 1> dt(a.dt, row, step, a.passing), o(a.o, row, step, a.passing);
  Stream<kType, kEnd, 1> dx(a.dx, row, step, a.passing), dout(a.dout, row, step, a.passing);
  float4 next;
  auto load = [&](int64_t r) {
    const bool here = r < a.rows;
    dh.load(c, here);
    t.load(c, here);
    dt.load(c, here);
    o.load(c, here);
    next = a.stats && here ? reinterpret_cast<const float4*>(a.stats)[r] : make_float4(0.f, 1.f, 0.f, 1.f);
  };
  load(row);
#pragma unroll
  for (int i = 0; i < (kBiases ? 4 : 3); ++i)
    if (i % groups == group)
      share_param(param_of(a, i), i < 3 ? 1.f : 0.f, shared_floats + i * 2 * lanes, lanes, lane, col, n);
  __syncthreads();
  auto param = [&](int i, float (&v)[8]) { shared_param(shared_floats + i * 2 * lanes, lanes, lane, v); };
  float total[kNormSums][8] = {};
  for (int64_t first = (int64_t)blockIdx.x * groups; first < a.rows; first += step, row += step) {
    const bool here = row < a.rows;
    float e[8], u[8], d[8], w[8], v[8];
    const float4 st = a.after.kind ? next : make_float4(0.f, 1.f, next.z, next.w);
    dh.values(0, c, e);
    t.values(0, c, u);
    dt.values(0, c, d);
    o.values(0, c, v);
    load(row + step);
    if (a.before.kind) {
      float se = 0.f, seu = 0.f;
      param(kBeforeWeight, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        u[i] = (u[i] - st.z) * st.w;
        total[0][i] += e[i] * u[i];
        if constexpr (kBiases) total[1][i] += e[i];
        e[i] *= w[i];
        se += e[i];
        seu += e[i] * u[i];
      }
      const bool layer = a.before.kind == POINTID_NORM_LAYER;
      const float2 s = layer ? row_sum(se, seu) : make_float2(0.f, row_sum(seu));
      const float on_u = st.w * (s.y * inv), on_1 = st.w * (s.x * inv);
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] += st.w * e[i] - on_u * u[i] - on_1;
      // columns and rows that do not exist add nothing
      zero_past(c.any_end[0], n, d);
      if (!here)
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = a.scale * d[i];
    dx.store(col, n, here, u);
    dx.next();
    if (!a.o.p && !a.dout.p) continue;
    if (a.drop.threshold) {
      if (a.after.kind)
        drop8(a.drop, key, row, col, d);
      else
        drop8(a.drop, key, row, col, d, &v);
    }
    param(kAfterWeight, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = (v[i] - st.x) * st.y;
      u[i] = v[i] * w[i];
    }
    if constexpr (kBiases) {
      float b[8];
      param(kAfterBias, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] += b[i];
    }
    float g[8];
    param(kGate, g);
    float sf = 0.f, sfv = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      total[4][i] += d[i] * u[i];
      d[i] *= g[i];
      total[2][i] += d[i] * v[i];
      if constexpr (kBiases) total[3][i] += d[i];
      d[i] *= w[i];
      sf += d[i];
      sfv += d[i] * v[i];
    }
    if (!a.dout.p) continue;
    if (a.after.kind) {
      const bool layer = a.after.kind == POINTID_NORM_LAYER;
      const float2 s = layer ? row_sum(sf, sfv) : make_float2(0.f, row_sum(sfv));
      const float on_v = st.y * (s.y * inv), on_1 = st.y * (s.x * inv);
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = st.y * d[i] - on_v * v[i] - on_1;
    }
    dout.store(col, n, here, d);
    dout.next();
  }
  // the groups' sums, in order; by halves, as the parameters stand
  int wanted = 0, slot = 0;
  for (int s = 0; s < kNormSums; ++s) wanted += a.out[s] != nullptr;
#pragma unroll
  for (int s = 0; s < kNormSums; ++s) {
    if (!a.out[s]) continue;
    float* const out = gridDim.x == 1 ? a.out[s] : a.part + ((int64_t)blockIdx.x * wanted + slot) * a.cols;
    ++slot;
    if (groups > 1) {
      __syncthreads();
      float4* const mine = shared_floats + group * 2 * lanes;
      mine[lane] = make_float4(total[s][0], total[s][1], total[s][2], total[s][3]);
      mine[lanes + lane] = make_float4(total[s][4], total[s][5], total[s][6], total[s][7]);
      __syncthreads();
      if (group != 0) continue;
      for (int g = 1; g < groups; ++g) {
        float v[8];
        shared_param(shared_floats + g * 2 * lanes, lanes, lane, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) total[s][i] += v[i];
      }
    }
    store_cols<8>(out, col, POINTID_FP32, n, total[s]);
  }
}

// The sums of the blocks' sums: 32 columns of one parameter a block, 32 of the partial rows
// at a time, added in order (256 rows of 3 x 4096: 4.8 us; 8 rows at a time 10).
__global__ void __launch_bounds__(1024) norm_sums_kernel(NormBackArgs a) {
  __shared__ float sums[32][33];
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
    for (int b = sub; b < a.blocks; b += 32) t += a.part[((int64_t)b * wanted + at) * a.cols + col];
  sums[sub][c] = t;
  __syncthreads();
  if (sub != 0 || col >= a.cols) return;
  t = 0.f;
#pragma unroll
  for (int s = 0; s < 32; ++s) t += sums[s][c];
  a.out[which][col] = t;
}

unsigned row_blocks(int64_t rows) { return (unsigned)(rows < 65536 ? rows : 65536); }

// Columns that a block can hold of a row, 8 a thread.
constexpr int64_t kHeldCols = 8192;
constexpr size_t kMostShared = 156 * 1024;     // of a CU's 160 KB, some taken by the sums' exchange
// Threads of a row that is held (16, or whole waves), and the groups of them in a block of at
// most `threads`, or one.
struct HeldShape {
  int lanes, groups;
};
HeldShape held_shape(int64_t cols, int threads) {
  const int lanes = cols <= 128 ? 16 : (int)((cols + 511) / 512) * 64;
  return {lanes, lanes < threads ? threads / lanes : 1};
}
// Threads of a block of the backward pass: 768 leave each 168 registers, which the sums of biases
// and fp32 rows take; 1024 leave 128.  768 and 1024: bf16 16384 x 4096 with biases 160 us and 235,
// fp32 8192 x 4096 without 166 and 175, bf16 300000 x 100 without 175 and 152.  Rows of more than 6144
// columns are a block of more threads, whose 128 registers do not hold these (22 to 40 of them in
// memory with biases, 6 to 8 without): in the two passes of wider rows they would take longer all the same.
// Held and in two passes, layer norms with biases, bf16 4096 x 8192 115 us and 185, 1693 x 7168 71 and 79,
// 4096 x 8191 175 and 329, fp32 4096 x 8192 257 and 304, 1693 x 7168 128 and 128; without, 181 and 300, 80 and 124.
int back_threads(int dtype, bool biases, int64_t cols) {
  return (biases || dtype == POINTID_FP32) && cols <= 6144 ? 768 : 1024;
}

// f with constants: whether a row has 16 threads, how it ends, whether there are biases.
template <class F>
hipError_t with_shape(int64_t cols, bool biases, F&& f) {
  auto up = [&](auto small, auto end) {
    return biases ? f(small, end, std::true_type{}) : f(small, end, std::false_type{});
  };
  const Which<kWhole> whole;
  const Which<kRagged> ragged;
  if (cols < 8) return up(std::true_type{}, Which<kTiny>{});
  if (cols <= 128) return cols % 8 ? up(std::true_type{}, ragged) : up(std::true_type{}, whole);
  return cols % 8 ? up(std::false_type{}, ragged) : up(std::false_type{}, whole);
}

template <int kType>
hipError_t launch_norm_of(NormArgs a, hipStream_t stream) {
  if (a.cols > 2 * kHeldCols) return launch_kernel(norm_kernel<kType>, dim3(row_blocks(a.rows)), dim3(256), 0, stream, a);
  const bool biases = a.after.bias || a.before.bias;
  const bool two = a.cols > kHeldCols;           // pieces a thread
  a.passing = passes_cache(kType, a.rows, a.cols, 1 + (a.o.p != nullptr) + (a.t.p != nullptr) + (a.h.p != nullptr));
  const HeldShape h = held_shape(two ? (a.cols + 1) / 2 : a.cols, 256);
  a.lanes = h.lanes;
  const int64_t need = (a.rows + h.groups - 1) / h.groups;
  // Many rows: blocks of at least 8 sets of rows, with the parameters in shared memory.  bf16, both
  // norms and a gate, read from memory for every row and shared: 16384 x 4096 121 us and 104, 8192 x
  // 4096 59 and 49, 8192 x 8192 150 and 105; fp32 8192 x 4096 113 and 104.  Few rows wait for the staging:
  // 3000 x 4096 23.5 us and 24.5, 4100 x 4096 30.7 and 28.4, 2100 x 8192 41 and 47, 4100 x 8192 78 and 58,
  // fp32 2100 x 4096 29 and 34, 4100 x 4096 53 and 49.
  const bool shared = need >= 4096 && !two;
  // Biases as well where they fit: five against three of five, both norms layer norms with biases and a
  // gate: bf16 16384 x 2304 80 us and 91, 16384 x 3200 (14 waves a CU) 106 and 111, 8192 x 5120 (10) 93 and
  // 96; but with 8 or 9 waves a CU too few loads are on their way: 16384 x 4096 154 and 106, 5280 x 4288 71
  // and 56.  fp32, whose loads are twice as large, 16384 x 4096 204 and 208, 5280 x 4288 79 and 88.
  auto bytes = [&](int params) { return (size_t)params * h.lanes * 32; };
  const int waves = (int)(kMostShared / bytes(5)) * (h.lanes * h.groups / 64);
  const bool five = biases && waves >= (kType == POINTID_FP32 ? 1 : 10);
  int64_t blocks = need < 65536 ? need : 65536;
  if (shared) blocks = need / 8 < 4096 ? need / 8 : 4096;
  auto go = [&](auto kernel, size_t shared_bytes) {
    return launch_kernel(kernel, dim3((unsigned)blocks), dim3(h.lanes * h.groups), shared_bytes, stream, a);
  };
  return with_shape(a.cols, biases, [&](auto small, auto end, auto bias) {
    if constexpr (bias)
      if (shared && five) return go(norm_rows_kernel<kType, small, end, bias, 5, 1>, bytes(5));
    if (shared) return go(norm_rows_kernel<kType, small, end, bias, 3, 1>, bytes(3));
    if constexpr (!small)
      if (two) return go(norm_rows_kernel<kType, false, end, bias, 0, 2>, 0);
    return go(norm_rows_kernel<kType, small, end, bias, 0, 1>, 0);
  });
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
  switch (a.dtype) {
    case POINTID_FP32: return launch_norm_of<POINTID_FP32>(a, stream);
    case POINTID_BF16: return launch_norm_of<POINTID_BF16>(a, stream);
  }
  return launch_norm_of<POINTID_FP16>(a, stream);
}

namespace {
bool has_biases(const NormBackArgs& a) { return a.out[1] || a.out[3] || a.after.bias; }
}  // namespace

NormBackPlan plan_norm_back(const NormBackArgs& a, int cus) {
  const int64_t rows = a.rows, cols = a.cols;
  NormBackPlan p;
  p.held = cols <= kHeldCols;
  if (p.held) {
    const int groups = held_shape(cols, back_threads(a.dtype, has_biases(a), cols)).groups;
    const int64_t need = (rows + groups - 1) / groups, most = cus;
    p.blocks = (int32_t)(need < most ? need : most);
  } else {
    const int64_t strips = (cols + 255) / 256, most = (rows + 31) / 32, want = (8 * cus + strips - 1) / strips;
    p.blocks = (int32_t)(most < want ? most : want);
  }
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

namespace {
template <int kType>
hipError_t launch_norm_back_of(NormBackArgs a, bool held, hipStream_t stream) {
  if (!held)
    return launch_kernel(norm_back_kernel<kType>, dim3((unsigned)((a.cols + 255) / 256), (unsigned)a.blocks), dim3(256), 0,
                         stream, a);
  int matrices = 0;
  for (const Rows* r : {&a.dh, &a.dt, &a.t, &a.o, &a.dx, &a.dout}) matrices += r->p != nullptr;
  a.passing = passes_cache(kType, a.rows, a.cols, matrices);
  const bool biases = has_biases(a);
  const int threads = back_threads(kType, biases, a.cols);
  const HeldShape h = held_shape(a.cols, threads);
  a.lanes = h.lanes;
  // the parameters, or the groups' sums: at most 128 KB
  const int shared = biases ? 4 : 3;
  return with_shape(a.cols, biases, [&](auto small, auto end, auto bias) {
    auto go = [&](auto kernel) {
      return launch_kernel(kernel, dim3((unsigned)a.blocks), dim3(h.lanes * h.groups),
                           (size_t)(shared > h.groups ? shared : h.groups) * h.lanes * 32, stream, a);
    };
    if constexpr (bias || kType == POINTID_FP32) {
      if constexpr (small) return go(norm_back_rows_kernel<kType, small, end, bias, 768>);
      if (threads == 768) return go(norm_back_rows_kernel<kType, small, end, bias, 768>);
    }
    if constexpr (!(small && (bias || kType == POINTID_FP32))) return go(norm_back_rows_kernel<kType, small, end, bias, 1024>);
  });
}
}  // namespace

hipError_t launch_norm_back(const NormBackArgs& a, bool held, hipStream_t stream) {
  switch (a.dtype) {
    case POINTID_FP32: return launch_norm_back_of<POINTID_FP32>(a, held, stream);
    case POINTID_BF16: return launch_norm_back_of<POINTID_BF16>(a, held, stream);
  }
  return launch_norm_back_of<POINTID_FP16>(a, held, stream);
}

hipError_t launch_norm_sums(const NormBackArgs& a, hipStream_t stream) {
  int wanted = 0;
  for (int s = 0; s < kNormSums; ++s) wanted += a.out[s] != nullptr;
  return launch_kernel(norm_sums_kernel, dim3((unsigned)((a.cols + 31) / 32), (unsigned)wanted), dim3(1024), 0, stream,
                       a);
}

}  // namespace pointid
