// Log probabilities of given columns, the log of the sum of exponentials, entropy and the most
// likely columns of each row of logits, and the logits' gradient.
//
// With z = scale x, m the row's maximum and d = z - m:
//   s = sum e^d    lse = m + ln s    logp(t) = d_t - ln s    H = ln s - (sum e^d d) / s
// Each thread keeps m, s and sum e^d d of the columns it has read (in powers of two: d / ln 2)
// and brings them to a new maximum when one comes, so that a row is read once.
//
// bf16 4096 x 65536 (537 MB) 100 us, 5.4 TB/s, with the 8 likeliest columns 112: near the bytes'
// time, and near the vector units' too, which are busy 80 % of it (an exponential is four instructions'
// time, and 6 more for each column are the difference, its scale, the clamp and the sums).
#include "internal.h"
#include "layers_end.h"
#include "norm.h"
#include "passing.h"
#include "wave.h"

namespace pointid {
namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
constexpr float kLowest = -3.402823466e38f;

// ---- the most likely columns.  An entry is 64 bits: above, the value's bits as an unsigned
// number in the order of the values; below, the column (or piece of 8 columns) inverted, so that
// among equals the lowest column is the largest entry.  0 is no entry.  A NaN counts as minus
// infinity, -0 as 0.
__device__ __forceinline__ uint32_t order_of(float v) {
  v = v != v ? -__builtin_inff() : v + 0.f;
  const uint32_t b = __float_as_uint(v);
  return b ^ ((int32_t)b < 0 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order) {
  return __uint_as_float(order ^ ((int32_t)order < 0 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ uint64_t entry_of(float v, uint32_t at) { return (uint64_t)order_of(v) << 32 | (uint32_t)~at; }

template <int kX>
__device__ __forceinline__ uint64_t entry_xor(uint64_t v) {
  return (uint64_t)lane_xor<kX>((uint32_t)(v >> 32)) << 32 | lane_xor<kX>((uint32_t)v);
}
template <int kX>
__device__ __forceinline__ uint32_t entry_xor(uint32_t v) {
  return lane_xor<kX>(v);
}
template <class T>
__device__ __forceinline__ T keep_one(T v, T other, bool larger) {
  return (v > other) == larger ? v : other;
}
// kFirst, kFirst / 2, .. 1 lanes apart: the last steps of a bitonic sort, each lane of which keeps
// the larger where it is the lower one of a falling stretch of kStretch lanes or the upper of a
// rising one
template <int kFirst, int kStretch, class T>
__device__ __forceinline__ T sort_steps(T v) {
  const int lane = threadIdx.x % 64;
  v = keep_one(v, entry_xor<kFirst>(v), ((lane & kFirst) == 0) == ((lane & kStretch) == 0));
  if constexpr (kFirst > 1) return sort_steps<kFirst / 2, kStretch>(v);
  return v;
}
// A wave's 64 entries in falling order (a bitonic sort), and the 64 largest of two such lists.
template <class T>
__device__ __forceinline__ T sort64(T v) {
  v = sort_steps<1, 2>(v);
  v = sort_steps<2, 4>(v);
  v = sort_steps<4, 8>(v);
  v = sort_steps<8, 16>(v);
  v = sort_steps<16, 32>(v);
  return sort_steps<32, 64>(v);
}
template <class T>
__device__ __forceinline__ T merge64(T a, T b) {
  b = entry_xor<63>(b);
  return sort_steps<32, 64>(a > b ? a : b);
}
// The 64 largest of the waves' lists, in the first wave.
template <int kWaves, class T>
__device__ __forceinline__ T merge_waves(T v, uint64_t (&lists)[kWaves > 1 ? kWaves / 2 * 64 : 1]) {
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
#pragma unroll
  for (int half = kWaves / 2; half > 0; half /= 2) {
    __syncthreads();
    if (wave >= half && wave < 2 * half) lists[(wave - half) * 64 + lane] = v;
    __syncthreads();
    if (wave < half) v = merge64(v, (T)lists[wave * 64 + lane]);
  }
  return v;
}

// The same entry of a 16-bit value and one of 65536 places in 32 bits, and back.
template <int kType>
__device__ __forceinline__ uint32_t short_entry(float v, uint32_t place) {
  const uint32_t b = to16(v + 0.f, kType);
  return (b ^ (b & 0x8000u ? 0xFFFFu : 0x8000u)) << 16 | (0xFFFFu - place);
}
template <int kType>
__device__ __forceinline__ uint64_t long_entry(uint32_t e, uint32_t first_place) {
  const uint32_t o = e >> 16, b = o ^ (o & 0x8000u ? 0x8000u : 0xFFFFu);
  return e == 0 ? 0 : entry_of(from16((uint16_t)b, kType), first_place + (0xFFFFu - (e & 0xFFFFu)));
}

// ---- maximum, sum of 2^d and of 2^d d of some columns, d = c (x - maximum) with c = scale / ln 2
// (the difference first: a column at the maximum adds 1 exactly)
struct Sums {
  float most, s, w;
};
// A result of `of`, fp32's largest finite value in place of an infinity that is not of's own.
__device__ __forceinline__ float in_range(float v, float of) {
  return __builtin_isinf(v) && !__builtin_isinf(of) ? __builtin_copysignf(-kLowest, v) : v;
}
// What is subtracted: finite, so that no infinity meets itself in a row that is masked whole.
__device__ __forceinline__ float finite_most(float most) { return fmaxf(most, kLowest); }
constexpr float kNone = -1000.f;               // 2^kNone is 0, and kNone times it too
// v brought to the maximum `most`, which is no smaller than its own.
__device__ __forceinline__ void bring_to(Sums* v, float most, float c) {
  const float d = fmaxf((finite_most(v->most) - finite_most(most)) * c, kNone), e = two_to(d);
  v->w = e * (v->w + d * v->s);
  v->s = e * v->s;
  v->most = most;
}
// 8 values: a NaN, or infinity less itself, stays a NaN; minus infinity adds nothing
template <bool kEntropy>
__device__ __forceinline__ void add_to(Sums* v, const float (&x)[8], float ref, float c) {
  float s = 0.f, w = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float d = (x[i] - ref) * c, e = two_to(d);
    s += e;
    if constexpr (kEntropy) w += e * fmaxf(d, kNone);
  }
  v->s += s;
  if constexpr (kEntropy) v->w += w;
}
__device__ __forceinline__ float max8(const float (&v)[8]) {
  return fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
}
// The same of values as they come, without the instruction that would quiet each one's signalling
// NaN first: one of these may lose what was the maximum before it.
__device__ __forceinline__ float max3_as_is(float a, float b, float c) {
  float m;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
  return m;
}
__device__ __forceinline__ float max8_as_is(const float (&v)[8]) {
  return max3_as_is(max3_as_is(max3_as_is(v[0], v[1], v[2]), v[3], v[4]), max3_as_is(v[5], v[6], v[7]), v[7]);
}

template <int kWaves>
__device__ __forceinline__ void block_sums(Sums* v, float c, float (&lds)[kWaves][2]) {
  float most = lanes_max<64>(v->most);
  const int wave = threadIdx.x / 64;
  if constexpr (kWaves > 1) {
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[wave][0] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaves; ++i) most = fmaxf(most, lds[i][0]);
  }
  bring_to(v, most, c);
  v->s = lanes_sum<64>(v->s);
  v->w = lanes_sum<64>(v->w);
  if constexpr (kWaves > 1) {
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[wave][0] = v->s, lds[wave][1] = v->w;
    __syncthreads();
    v->s = lds[0][0], v->w = lds[0][1];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) v->s += lds[i][0], v->w += lds[i][1];
  }
}

// A row's results from its sums: by any thread.
struct RowEnd {
  float most, scale, ln_s, lse, entropy;
  bool empty;                  // every column is masked
  __device__ __forceinline__ RowEnd(const Sums& v, float scale_) : most(v.most), scale(scale_) {
    empty = v.s == 0.f;
    ln_s = logf(v.s);
    // (past fp32's range its end: minus infinity is a row of nothing alone)
    lse = empty ? -__builtin_inff() : in_range(most * scale + ln_s, most);
    entropy = empty ? 0.f : ln_s - kLn2 * v.w / v.s;
  }
  // (halves: the difference of the range's ends is past it, scale times it need not be)
  __device__ __forceinline__ float logp(float x) const {
    return empty ? -__builtin_inff() : (0.5f * x - 0.5f * most) * (2.f * scale) - ln_s;
  }
};
__device__ __forceinline__ void store_row(const ScanArgs& a, int64_t row, const RowEnd& end, bool has_target, float target) {
  if (a.logp) a.logp[row] = has_target ? end.logp(target) : 0.f;
  if (a.lse) a.lse[row] = end.lse;
  if (a.entropy) a.entropy[row] = end.entropy;
}
__device__ __forceinline__ void store_top(const ScanArgs& a, int64_t row, const RowEnd& end, int at, uint64_t entry) {
  a.top_ids[row * a.top + at] = (int32_t)~(uint32_t)entry;
  a.top_logp[row * a.top + at] = end.logp(value_of((uint32_t)(entry >> 32)));
}

constexpr int kListed = 512;   // candidates that shared memory holds

// The k largest entries of columns [first, last) of a row, in falling order in the first wave's
// lanes.  The largest entry of each thread's own pieces (first / 8 + thread + i kThreads), by
// piece, is 0 of none (made of top, its value, and the place of the piece, past the first: sorted
// in 32 bits where the type has 16).  The columns that are wanted are all in pieces of the threads with the k
// largest of these: of any other thread, k threads have a larger one.  So those threads' pieces
// are read again, and what is at least the k-th of the threads' best is listed; more than the
// list holds (which takes an order of the values that goes with the threads') is sorted as it
// is read.
template <int kType, int kThreads>
__device__ uint64_t pick_top(const char* x, int64_t first, int64_t last, int k, float top, uint32_t place,
                             uint64_t (&lists)[kThreads > 64 ? kThreads / 128 * 64 : 1], uint64_t (&listed)[kListed],
                             uint32_t* count) {
  constexpr int kWaves = kThreads / 64, kSize = kType == POINTID_FP32 ? 4 : 2;
  __shared__ uint64_t chosen[kMaxTop];
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const bool any = first + threadIdx.x * 8 < last;
  uint64_t best;
  bool sorted = false;
  if constexpr (kType != POINTID_FP32) {
    if (last - first <= 65536 * 8) {
      const uint32_t e = any ? short_entry<kType>(top, place) : 0;
      best = long_entry<kType>(merge_waves<kWaves>(sort64(e), lists), (uint32_t)(first / 8));
      sorted = true;
    }
  }
  if (!sorted) best = merge_waves<kWaves>(sort64(any ? entry_of(top, (uint32_t)(first / 8) + place) : 0), lists);
  __syncthreads();
  if (threadIdx.x < (unsigned)k) chosen[threadIdx.x] = best;
  if (threadIdx.x == 0) *count = 0;
  __syncthreads();
  int threads = k;
  while (threads > 0 && chosen[threads - 1] == 0) --threads;   // fewer have any columns
  const uint64_t least = threads == k ? chosen[k - 1] : 0;
  const uint32_t base = (uint32_t)(first / 8), pieces = (uint32_t)((last + 7) / 8);
  const uint32_t each = (pieces - base + kThreads - 1) / kThreads;
  // whether an entry by column is at least `least`, by piece
  auto wanted = [&](uint64_t e) {
    return (e >> 32) > (least >> 32) || ((e >> 32) == (least >> 32) && (~(uint32_t)e) / 8 <= ~(uint32_t)least);
  };
  for (uint32_t i = threadIdx.x; i < threads * each; i += kThreads) {
    const uint32_t of = ~(uint32_t)chosen[i / each], piece = base + (of - base) % kThreads + i % each * kThreads;
    if (piece >= pieces) continue;
    Raw8<kType> raw;
    const int64_t col = (int64_t)piece * 8;
    const int n = piece_cols(last, col);
    raw.load(x + col * kSize, n);
    float v[8];
    raw.values(v);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= n) continue;
      const uint64_t e = entry_of(v[j], (uint32_t)col + j);
      if (!wanted(e)) continue;
      const uint32_t at = atomicAdd(count, 1);   // in any order: they are sorted, and no two are equal
      if (at < kListed) listed[at] = e;
    }
  }
  __syncthreads();
  const uint32_t found = *count;
  uint64_t v = 0;
  if (found <= kListed) {
    for (uint32_t at = wave * 64; at < found; at += kThreads) {
      const uint64_t e = sort64(at + lane < found ? listed[at + lane] : 0);
      v = at == (uint32_t)wave * 64 ? e : merge64(v, e);
    }
  } else {
    const uint32_t total = threads * each * 8;
    for (uint32_t at = wave * 64; at < total; at += kThreads) {
      uint64_t e = 0;
      const uint32_t i = (at + lane) / 8, j = lane % 8;
      if (i < threads * each) {
        const uint32_t of = ~(uint32_t)chosen[i / each], piece = base + (of - base) % kThreads + i % each * kThreads;
        const int64_t col = (int64_t)piece * 8 + j;
        if (piece < pieces && col < last) e = entry_of(load_any(x, col, kType), (uint32_t)col);
        if (!wanted(e)) e = 0;
      }
      if (__any(e != 0)) v = merge64(v, sort64(e));
    }
  }
  if (found <= 64) return v;                   // all in the first wave's list
  return merge_waves<kWaves>(v, lists);
}

// A row (or a split of one) by a block.  kAhead pieces of 8 columns a thread are brought to a new
// maximum at once, while the next are on their way.
template <int kType, int kThreads, bool kEntropy>
__global__ void __launch_bounds__(kThreads) scan_kernel(ScanArgs a) {
  constexpr int kSize = kType == POINTID_FP32 ? 4 : 2, kWaves = kThreads / 64, kAhead = 2;
  __shared__ float lds[kWaves][2];
  __shared__ uint64_t lists[kThreads > 64 ? kThreads / 128 * 64 : 1], listed[kListed];
  __shared__ uint32_t count;
  const float c = a.scale * kLog2e;
  for (int64_t unit = blockIdx.x; unit < a.rows * a.splits; unit += gridDim.x) {
    const int64_t row = a.splits == 1 ? unit : unit / a.splits, split = unit - row * a.splits;
    const int64_t first = split * a.split_cols;
    const int64_t last = first + a.split_cols < a.cols ? first + a.split_cols : a.cols;
    const char* const x = a.x.p + row * a.x.ld * kSize;
    const int mine = (int)threadIdx.x * 8, width = (int)(last - first);
    Sums v = {-__builtin_inff(), 0.f, 0.f};
    float top = -__builtin_inff();
    uint32_t top_turn = 0;
    const char* const at = x + first * kSize;
    // turns of kAhead pieces a thread; those that are whole for every thread, and one more
    constexpr int kTurn = kThreads * 8 * kAhead;
    const int whole = width / kTurn, turns = (width + kTurn - 1) / kTurn;
    auto load = [&](Raw8<kType> (&raw)[kAhead], int turn) {
      const char* const p = at + ((int64_t)turn * kTurn + mine) * kSize;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (turn < whole)
          raw[u].load(p + u * kThreads * 8 * kSize, 8);
        else
          raw[u].load(p + u * kThreads * 8 * kSize, piece_cols(width, turn * kTurn + u * kThreads * 8 + mine));
      }
    };
    auto take = [&](const Raw8<kType> (&raw)[kAhead], int turn) {
      float f[kAhead][8];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) raw[u].values(f[u]);
      if (turn >= whole) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int n = piece_cols(width, turn * kTurn + u * kThreads * 8 + mine);
#pragma unroll
          for (int i = 0; i < 8; ++i) f[u][i] = i < n ? f[u][i] : -__builtin_inff();
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const float m = max8_as_is(f[u]);
        top_turn = m > top ? turn * kAhead + u : top_turn;
        top = max3_as_is(top, m, m);
      }
      if (top > v.most) bring_to(&v, top, c);
      const float ref = finite_most(top);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) add_to<kEntropy>(&v, f[u], ref, c);
    };
    // two sets of registers in turn
    Raw8<kType> raw[kAhead], ahead[kAhead];
    load(raw, 0);
    for (int turn = 0; turn < turns; turn += 2) {
      if (turn + 1 < turns) load(ahead, turn + 1);
      take(raw, turn);
      if (turn + 1 >= turns) break;
      if (turn + 2 < turns) load(raw, turn + 2);
      take(ahead, turn + 1);
    }
    if (v.s != v.s) {
      // a NaN: its columns' maximum again, NaNs left out
      top = -__builtin_inff(), top_turn = 0;
      for (int i = 0; mine + i * kThreads * 8 < width; ++i) {
        Raw8<kType> one;
        const int n = piece_cols(width, mine + i * kThreads * 8);
        one.load(at + (int64_t)(mine + i * kThreads * 8) * kSize, n);
        float f[8];
        one.values(f);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = k < n ? f[k] : -__builtin_inff();
        const float m = max8(f);
        top_turn = m > top ? i : top_turn;
        top = fmaxf(top, m);
      }
      v.most = top;
    }
    block_sums<kWaves>(&v, c, lds);
    uint64_t entry = 0;
    if (a.top) {
      entry = pick_top<kType, kThreads>(x, first, last, a.top, top, threadIdx.x + top_turn * kThreads, lists, listed, &count);
    }
    if (a.splits > 1) {
      if (threadIdx.x == 0) reinterpret_cast<float4*>(a.part)[unit] = make_float4(v.most, v.s, v.w, 0.f);
      if (threadIdx.x < (unsigned)a.top) a.part_top[unit * a.top + threadIdx.x] = entry;
      continue;
    }
    const RowEnd end(v, a.scale);
    if (threadIdx.x == 0) {
      const int32_t t = a.targets ? a.targets[row] : -1;
      const bool has = t >= 0 && t < a.cols;
      store_row(a, row, end, has, has ? load_any(x, t, kType) : 0.f);
    }
    if (threadIdx.x < (unsigned)a.top) store_top(a, row, end, threadIdx.x, entry);
  }
}

// Rows of at most 8 kLanes columns, each by kLanes lanes that hold 8 of them; the most likely
// columns one by one, each a pass over the row's lanes.  fp32 50000 x 3 with the likeliest: 3.5 us (a block a
// row: 280); bf16 500000 x 64 (64 MB) with 0, 1 and 20 of them 20, 30 and 125, 50000 x 500 with 0, 1, 8
// and 32 23, 30, 58 and 158.
template <int kType, int kLanes>
__global__ void __launch_bounds__(256) scan_short_kernel(ScanArgs a) {
  constexpr int kSize = kType == POINTID_FP32 ? 4 : 2, kRows = 256 / kLanes;
  const float c = a.scale * kLog2e;
  const int lane = threadIdx.x % kLanes, col = lane * 8, n = piece_cols(a.cols, col);
  for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < a.rows; row0 += (int64_t)gridDim.x * kRows) {
    const int64_t row = row0 + threadIdx.x / kLanes;
    if (row >= a.rows) continue;
    const char* const x = a.x.p + row * a.x.ld * kSize;
    const int32_t target = a.targets ? a.targets[row] : -1;
    Raw8<kType> raw;
    raw.load(x + col * kSize, n);
    float f[8];
    raw.values(f);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? f[i] : -__builtin_inff();
    Sums v = {lanes_max<kLanes>(max8(f)), 0.f, 0.f};
    add_to<true>(&v, f, finite_most(v.most), c);
    v.s = lanes_sum<kLanes>(v.s);
    v.w = lanes_sum<kLanes>(v.w);
    const RowEnd end(v, a.scale);
    const bool has = target >= 0 && target < a.cols;
    if (has ? target / 8 == lane : lane == 0) {
      float t = f[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) t = target % 8 == i ? f[i] : t;
      store_row(a, row, end, has, t);
    }
    if (a.top == 0) continue;
    uint32_t order[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) order[i] = i < n ? order_of(f[i]) : 0;
    for (int k = 0; k < a.top; ++k) {
      uint32_t best = 0;
      int at = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        at = order[i] > best ? i : at;
        best = order[i] > best ? order[i] : best;
      }
      const uint32_t most = over_lanes<kLanes>(best, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
      // the first lane of the row's that has it
      bool mine = best == most;
      if constexpr (kLanes > 1) {
        const uint64_t same = __ballot(mine) >> (threadIdx.x % 64 / kLanes * kLanes);
        mine = __builtin_ctzll(same) == lane;
      }
      if (mine) {
        store_top(a, row, end, k, (uint64_t)best << 32 | (uint32_t)~(col + at));
#pragma unroll
        for (int i = 0; i < 8; ++i) order[i] = at == i ? 0 : order[i];
      }
    }
  }
}

// The splits of a row joined, by a block: 6 us for 32 splits' lists of 20 (1 x 131072, whose scan
// takes 7).
template <int kType>
__global__ void __launch_bounds__(512) scan_join_kernel(ScanArgs a) {
  constexpr int kWaves = 8;
  __shared__ float lds[kWaves][2];
  __shared__ uint64_t lists[kWaves / 2 * 64];
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const float c = a.scale * kLog2e;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    Sums v = {-__builtin_inff(), 0.f, 0.f};
    for (int s = threadIdx.x; s < a.splits; s += kWaves * 64) {
      const float4 p = reinterpret_cast<const float4*>(a.part)[row * a.splits + s];
      Sums other = {p.x, p.y, p.z};
      const float most = fmaxf(v.most, other.most);
      bring_to(&v, most, c);
      bring_to(&other, most, c);
      v.s += other.s;
      v.w += other.w;
    }
    block_sums<kWaves>(&v, c, lds);
    uint64_t entry = 0;
    if (a.top) {
      for (int s = wave; s < a.splits; s += kWaves)
        entry = merge64(entry, lane < a.top ? a.part_top[(row * a.splits + s) * a.top + lane] : 0);
      entry = merge_waves<kWaves>(entry, lists);
    }
    const RowEnd end(v, a.scale);
    if (threadIdx.x == 0) {
      const int32_t t = a.targets ? a.targets[row] : -1;
      const bool has = t >= 0 && t < a.cols;
      store_row(a, row, end, has, has ? load_any(a.x.p, row * a.x.ld + t, kType) : 0.f);
    }
    if (threadIdx.x < (unsigned)a.top) store_top(a, row, end, threadIdx.x, entry);
  }
}

// dx_j = scale (dlogp ([j = t] - p_j) + dlse p_j - dH p_j (ln p_j + H)), p_j = e^(z_j - lse), as
//   q = log2 p_j = x_j scale / ln 2 - lse / ln 2       dx_j = 2^q (on_p - on_pq q) + [j = t] at_target
// x scale, rounded and in fp32's range, less lse
__device__ __forceinline__ float rounded_less(float x, float scale, float lse) {
#pragma clang fp contract(off)
  const float z = in_range(x * scale, x);
  return z - lse;
}
struct BackRow {
  float lse, lse2, at_target, on_p, on_pq;
  int32_t target;
  bool far;                    // lse is large: see gradient
  // what is read of a row; kept until its turn
  struct Read {
    float lse, dlogp, dlse, dh, h;
    int32_t target;
    __device__ __forceinline__ void load(const ScanBackArgs& a, int64_t row, bool here) {
      lse = here ? a.lse[row] : 0.f;
      target = here && a.targets ? a.targets[row] : -1;
      dlogp = here && a.dlogp ? a.dlogp[row] : 0.f;
      dlse = here && a.dlse ? a.dlse[row] : 0.f;
      dh = here && a.dentropy ? a.dentropy[row] : 0.f;
      h = here && a.dentropy ? a.entropy[row] : 0.f;
    }
  };
  __device__ __forceinline__ BackRow(const Read& r, float scale, int64_t cols) {
    const bool empty = r.lse == -__builtin_inff(), has = r.target >= 0 && r.target < cols && !empty;
    target = has ? r.target : -1;
    at_target = has ? r.dlogp * scale : 0.f;
    // (of a row of nothing 0, as a loss may make an infinity or a NaN of its lse)
    on_p = empty ? 0.f : r.dlse * scale - at_target - r.dh * r.h * scale;
    on_pq = empty ? 0.f : r.dh * scale * kLn2;
    lse = empty ? __builtin_inff() : r.lse;                   // p is 0 in a row of nothing
    lse2 = lse * kLog2e;
    far = !empty && __builtin_fabsf(lse) > 1024.f;
  }
  // (fp32: the difference first too, which the roundings of scale / ln 2 and lse / ln 2 are in
  // otherwise: they double the error of a result that is rounded to 24 bits.  Of a large lse, whose
  // own rounding passes that of p, z_j is rounded as the forward pass rounds the largest: what of it
  // lse cannot hold would be all that is left of the difference, and p past 1, by 2^60 in a bf16 row
  // of -1e9 alone.)
  template <int kType, bool kEntropy>
  __device__ __forceinline__ void gradient(float scale, float c, int col, float (&v)[8]) const {
    if (far) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = rounded_less(v[j], scale, lse) * kLog2e;
    } else if (kType == POINTID_FP32) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __builtin_fmaf(v[j], scale, -lse) * kLog2e;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __builtin_fmaf(v[j], c, -lse2);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = two_to(v[j]) * (kEntropy ? on_p - on_pq * fmaxf(v[j], kNone) : on_p);
    const uint32_t at = (uint32_t)(target - col);
    if (at < 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += (uint32_t)j == at ? at_target : 0.f;
    }
  }
};

// A strip of 8 columns a thread, row after row: a block's threads are groups of `lanes` (kSmall: a
// part of a wave, else whole ones), each group with a row at a time, the next row on its way.
// bf16 4096 x 65536 with an entropy term (1.07 GB) 174 us, 6.2 TB/s; as pieces of any row, whose place
// is a division and whose row's values are read for each piece, 200 and the vector units busy 86 %, now 72.
// Rows of 33 to 63 pieces leave lanes of a wave without one, and a row's end inside a piece is read and
// written value by value: bf16 100000 x 300 43 us, x 303 49, x 304 32, x 1000 77 (5.2 TB/s).
template <int kType, bool kSmall, bool kEntropy>
__global__ void __launch_bounds__(256) scan_back_kernel(ScanBackArgs a) {
  constexpr int64_t kSize = kType == POINTID_FP32 ? 4 : 2;
  const int lanes = a.lanes, groups = blockDim.x / lanes;
  const int group = kSmall ? (int)threadIdx.x / lanes : __builtin_amdgcn_readfirstlane((int)threadIdx.x / lanes);
  const int col = ((int)blockIdx.x * lanes + (int)threadIdx.x - group * lanes) * 8, n = piece_cols(a.cols, col);
  const float c = a.scale * kLog2e;
  const int64_t step = (int64_t)gridDim.y * groups;
  int64_t row = (int64_t)blockIdx.y * groups + group;
  const char* x = a.x.p + row * a.x.ld * kSize;
  char* dx = a.dx.p + row * a.dx.ld * kSize;
  Raw8<kType> raw;
  BackRow::Read read;
  auto load = [&](int64_t r) {
    Passing<kType>::load(&raw, x + col * kSize, r < a.rows ? n : 0, a.passing);
    read.load(a, r, r < a.rows);
    x += step * a.x.ld * kSize;
  };
  load(row);
  for (; row < a.rows; row += step) {
    float v[8];
    raw.values(v);
    const BackRow of(read, a.scale, a.cols);
    load(row + step);
    of.gradient<kType, kEntropy>(a.scale, c, col, v);
    if (n > 0) Passing<kType>::store(dx + col * kSize, n, v, a.passing);
    dx += step * a.dx.ld * kSize;
  }
}

}  // namespace

// Splits of a row, where the rows alone leave CUs idle: of at least 4096 columns.
int32_t scan_splits(int64_t rows, int64_t cols, int cus) {
  const int64_t most = (cols + 4095) / 4096, want = (2 * cus + rows - 1) / (rows > 0 ? rows : 1);
  const int64_t s = most < want ? most : want;
  return (int32_t)(s < 1 ? 1 : s);
}

namespace {
unsigned capped(int64_t blocks) { return (unsigned)(blocks < 65536 ? (blocks > 0 ? blocks : 1) : 65536); }
}  // namespace

namespace {
template <int kType>
hipError_t launch_logprobs_of(const ScanArgs& a, hipStream_t stream) {
  auto few = [&](auto kernel, int lanes) {
    return launch_kernel(kernel, dim3(capped((a.rows * lanes + 255) / 256)), dim3(256), 0, stream, a);
  };
  if (a.cols <= 8) return few(scan_short_kernel<kType, 1>, 1);
  if (a.cols <= 16) return few(scan_short_kernel<kType, 2>, 2);
  if (a.cols <= 32) return few(scan_short_kernel<kType, 4>, 4);
  if (a.cols <= 64) return few(scan_short_kernel<kType, 8>, 8);
  if (a.cols <= 128) return few(scan_short_kernel<kType, 16>, 16);
  if (a.cols <= 256) return few(scan_short_kernel<kType, 32>, 32);
  if (a.cols <= 512) return few(scan_short_kernel<kType, 64>, 64);
  auto go = [&](auto kernel, int threads) {
    return launch_kernel(kernel, dim3(capped(a.rows * a.splits)), dim3(threads), 0, stream, a);
  };
  // By waves of their own up to 8192 columns, where the rows fill the card so: a block's waves wait
  // for each other in the choice of the likeliest columns.  With the 8 likeliest, bf16, by waves and
  // by blocks of 4: 32768 x 4096 80 us and 228, 16384 x 8192 73-79 and 114, 16384 x 16384 171 and
  // 152, 4096 x 65536 169 and 120; 4096 x 8192 22 and 29, 4096 x 4096 12.4 and 23.5, 2048 x 8192 12.3 and
  // 15.6, of 1100 rows of 4096 or 8192 both less than the call's host side (11.6).  Without a list they are
  // alike from 4096 rows of 8192 on (16, 8192 rows 31), and of 4096 columns 9.3 and 10.4.
  if (a.cols <= 8192 && a.rows > 1024)
    return a.entropy ? go(scan_kernel<kType, 64, true>, 64) : go(scan_kernel<kType, 64, false>, 64);
  return a.entropy ? go(scan_kernel<kType, 256, true>, 256) : go(scan_kernel<kType, 256, false>, 256);
}
}  // namespace

hipError_t launch_logprobs(const ScanArgs& a, hipStream_t stream) {
  switch (a.dtype) {
    case POINTID_FP32: return launch_logprobs_of<POINTID_FP32>(a, stream);
    case POINTID_BF16: return launch_logprobs_of<POINTID_BF16>(a, stream);
  }
  return launch_logprobs_of<POINTID_FP16>(a, stream);
}

hipError_t launch_logprobs_join(const ScanArgs& a, hipStream_t stream) {
  const dim3 grid(capped(a.rows));
  switch (a.dtype) {
    case POINTID_FP32: return launch_kernel(scan_join_kernel<POINTID_FP32>, grid, dim3(512), 0, stream, a);
    case POINTID_BF16: return launch_kernel(scan_join_kernel<POINTID_BF16>, grid, dim3(512), 0, stream, a);
  }
  return launch_kernel(scan_join_kernel<POINTID_FP16>, grid, dim3(512), 0, stream, a);
}

hipError_t launch_logprobs_back(ScanBackArgs a, hipStream_t stream) {
  a.passing = passes_cache(a.dtype, a.rows, a.cols, 2);
  // A row's threads, of a block of 256: a power of two up to 32, then whole waves; and two sets of
  // rows a block, the second on its way beside the first: bf16 with entropy, one, two and four sets a
  // block, 4096 x 65536 210, 176 and 193 us, 16384 x 4096 56, 44 and 44, 32768 x 2048 57, 45 and 45.
  const int64_t pieces = (a.cols + 7) / 8;
  a.lanes = 1;
  while (a.lanes < 32 && a.lanes < pieces) a.lanes *= 2;
  const bool small = a.lanes >= pieces;
  if (!small) a.lanes = pieces <= 192 ? (int)(pieces + 63) / 64 * 64 : 256;
  const int groups = 256 / a.lanes;
  const int64_t strips = (pieces + a.lanes - 1) / a.lanes, sets = (a.rows + groups - 1) / groups;
  const dim3 grid((unsigned)strips, (unsigned)(sets < 2 * 65535 ? (sets + 1) / 2 : 65535));
  auto go = [&](auto type) {
    constexpr int kType = decltype(type)::value;
    auto run = [&](auto kernel) { return launch_kernel(kernel, grid, dim3(a.lanes * groups), 0, stream, a); };
    if (small) return a.dentropy ? run(scan_back_kernel<kType, true, true>) : run(scan_back_kernel<kType, true, false>);
    return a.dentropy ? run(scan_back_kernel<kType, false, true>) : run(scan_back_kernel<kType, false, false>);
  };
  switch (a.dtype) {
    case POINTID_FP32: return go(std::integral_constant<int, POINTID_FP32>{});
    case POINTID_BF16: return go(std::integral_constant<int, POINTID_BF16>{});
  }
  return go(std::integral_constant<int, POINTID_FP16>{});
}

}  // namespace pointid
