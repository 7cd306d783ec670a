// Device parts that the layer kernels share: types, activations, the 8-bit block
// format, and the end of a product (bias, activation, product of the halves, residual,
// kept activations).
#pragma once

#include "layers.h"
#include "op16.h"

namespace pointid {

__device__ __forceinline__ uint16_t to16(float v, int dtype) {
  if (dtype == POINTID_FP16) return __builtin_bit_cast(uint16_t, (_Float16)v);
  return __builtin_bit_cast(uint16_t, (__bf16)v);
}
__device__ __forceinline__ float from16(uint16_t h, int dtype) {
  if (dtype == POINTID_FP16) return (float)__builtin_bit_cast(_Float16, h);
  return __uint_as_float((uint32_t)h << 16);
}
__device__ __forceinline__ uint32_t pack16(float a, float b, int dtype) {
  return dtype == POINTID_FP16 ? Op16<true>::pack(a, b) : Op16<false>::pack(a, b);
}

__device__ __forceinline__ float load_any(const void* p, int64_t at, int dtype) {
  if (dtype == POINTID_FP32) return static_cast<const float*>(p)[at];
  return from16(static_cast<const uint16_t*>(p)[at], dtype);
}
__device__ __forceinline__ void store_any(void* p, int64_t at, float v, int dtype) {
  if (dtype == POINTID_FP32)
    static_cast<float*>(p)[at] = v;
  else
    static_cast<uint16_t*>(p)[at] = to16(v, dtype);
}

// kN (4, 8 or 16) consecutive values of a row, of which the first `n` exist; the rest
// read as 0 and are not written.  Pieces of 16 bytes at any alignment (the hardware
// takes them; aligned ones are faster).
template <int kN>
__device__ __forceinline__ void load_cols(const void* p, int64_t at, int dtype, int64_t n, float* v) {
  if (n >= kN) {
    if (dtype == POINTID_FP32) {
      __builtin_memcpy(v, static_cast<const float*>(p) + at, 4 * kN);
    } else {
      uint32_t w[kN / 2];
      __builtin_memcpy(w, static_cast<const uint16_t*>(p) + at, 2 * kN);
#pragma unroll
      for (int i = 0; i < kN / 2; ++i) {
        v[2 * i] = from16((uint16_t)w[i], dtype);
        v[2 * i + 1] = from16((uint16_t)(w[i] >> 16), dtype);
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kN; ++i) v[i] = i < n ? load_any(p, at + i, dtype) : 0.f;
}
template <int kN>
__device__ __forceinline__ void store_cols(void* p, int64_t at, int dtype, int64_t n, const float* v) {
  if (n >= kN) {
    if (dtype == POINTID_FP32) {
      __builtin_memcpy(static_cast<float*>(p) + at, v, 4 * kN);
    } else {
      uint32_t w[kN / 2];
#pragma unroll
      for (int i = 0; i < kN / 2; ++i) w[i] = pack16(v[2 * i], v[2 * i + 1], dtype);
      __builtin_memcpy(static_cast<uint16_t*>(p) + at, w, 2 * kN);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kN; ++i)
    if (i < n) store_any(p, at + i, v[i], dtype);
}

// ---- activations (fp32), from the hardware's 2^x and 1 / x (each within an ulp).
// sigmoid is off by at most 3e-7 + 1e-7 |z| of itself (measured: 1.4e-7 at 0, 0.7 of the bound
// at -85).  Phi, the normal distribution function, is Hastings' approximation of erfc
// (Abramowitz and Stegun 7.1.26), off by 7.5e-8 and the roundings of its terms, 3.1e-7 as
// measured; below -3, where Phi itself is small, by 7e-8.
// A NaN passes through all of them; relu's slope at 0 is 0.
__device__ __forceinline__ float two_to(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + two_to(-1.44269504088896341f * z));
}
// density: e^(-z^2 / 2)
__device__ __forceinline__ float normal_below(float z, float* density) {
  const float e = two_to(-0.72134752044448170f * z * z);
  const float t = __builtin_amdgcn_rcpf(1.f + 0.3275911f * 0.70710678118654752f * __builtin_fabsf(z));
  const float q = 0.5f * e * t *
                  (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
  *density = e;
  return z < 0.f ? q : 1.f - q;
}
__device__ __forceinline__ float activate(int act, float z) {
  float e;
  switch (act) {
    case POINTID_ACT_RELU: return z <= 0.f ? 0.f : z;
    case POINTID_ACT_SILU: return z * sigmoid(z);
    case POINTID_ACT_GELU: return z * normal_below(z, &e);
    case POINTID_ACT_SIGMOID: return sigmoid(z);
  }
  return z;
}
__device__ __forceinline__ void activate8(int act, float* v) {
  static_for<5>([&](auto a) {                 // the choice outside of the loop
    if (a != POINTID_ACT_NONE && act == a)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = activate(a, v[i]);
  });
}
// act(z), and the gradient d of it brought to z: d act'(z).  relu selects, so that an
// infinity or NaN does not get through where it is off.
__device__ __forceinline__ float through(int act, float z, float d, float* value) {
  float e;
  switch (act) {
    case POINTID_ACT_RELU:
      *value = z <= 0.f ? 0.f : z;
      return z <= 0.f ? 0.f : d;
    case POINTID_ACT_SILU: {
      const float s = sigmoid(z);
      *value = z * s;
      return d * (s * (1.f + z * (1.f - s)));
    }
    case POINTID_ACT_GELU: {
      const float below = normal_below(z, &e);
      *value = z * below;
      return d * (below + z * e * 0.39894228040143268f);
    }
    case POINTID_ACT_SIGMOID: {
      const float s = sigmoid(z);
      *value = s;
      return d * (s * (1.f - s));
    }
  }
  *value = z;
  return d;
}

// ---- the 8-bit block format.  The values of a block of 32 are multiplied by 2^p, p
// the largest integer with max |v| 2^p <= 448 (at most 126; 0 for a block of zeros), and
// rounded to e4m3 (nearest even); 127 - p is stored.  A value that is not finite is
// stored as NaN and does not count for the maximum.
__device__ __forceinline__ uint32_t finite_bits(float v) {
  const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}
__device__ __forceinline__ int block_power(uint32_t max_bits) {
  if (max_bits == 0) return 0;
  const float a = __uint_as_float(max_bits);             // f 2^e, f in [1/2, 1); 448 = 7/8 2^9
  const int e = __builtin_amdgcn_frexp_expf(a);
  const int p = __builtin_amdgcn_frexp_mantf(a) <= 0.875f ? 9 - e : 8 - e;
  return p < 126 ? p : 126;
}
__device__ __forceinline__ float scaled_for_8(float v, int p) {
  return (__float_as_uint(v) & 0x7FFFFFFFu) < 0x7F800000u ? __builtin_amdgcn_ldexpf(v, p) : __uint_as_float(0x7FC00000u);
}
__device__ __forceinline__ uint32_t pack8(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
__device__ __forceinline__ void unpack8(uint32_t w, int p, float* v) {       // times 2^p
  const floatx2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const floatx2 b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  v[0] = __builtin_amdgcn_ldexpf(a[0], p);
  v[1] = __builtin_amdgcn_ldexpf(a[1], p);
  v[2] = __builtin_amdgcn_ldexpf(b[0], p);
  v[3] = __builtin_amdgcn_ldexpf(b[1], p);
}

// 8 values of a row (of which the first n exist) to a checkpoint's codes at `c`, and by the
// first lane of a block its exponent to `x`.  The 4 lanes of an aligned group hold a block
// of 32 and all call this; values that do not exist do not count and are not written.
// `live`: the row and the first column exist.
__device__ __forceinline__ void save_codes(uint8_t* c, uint8_t* x, bool live, bool first, int n, const float* v) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = i < n ? finite_bits(v[i]) : 0u;
    top = b > top ? b : top;
  }
  uint32_t other = (uint32_t)__shfl_xor((int)top, 1, 64);
  top = other > top ? other : top;
  other = (uint32_t)__shfl_xor((int)top, 2, 64);
  top = other > top ? other : top;
  const int p = block_power(top);
  if (!live) return;
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    w[i] = pack8(scaled_for_8(v[4 * i], p), scaled_for_8(v[4 * i + 1], p), scaled_for_8(v[4 * i + 2], p),
                 scaled_for_8(v[4 * i + 3], p));
  if (n >= 8) {
    __builtin_memcpy(c, w, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) c[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
  if (first) *x = (uint8_t)(127 - p);
}

// Where 8 columns of a row of a result go; moved down by whole rows without multiplying.
template <int kType>
struct Target {
  static constexpr int kSize = kType == POINTID_FP32 ? 4 : 2;
  char* y;
  char* kept;                    // the matrix or the codes
  uint8_t* exponent;

  static __device__ __forceinline__ int64_t blocks(int64_t cols) { return (cols + kBlock8 - 1) / kBlock8; }
  __device__ __forceinline__ void init(void* out, int64_t ld, const Kept& k, int64_t cols, int64_t row, int64_t col) {
    y = static_cast<char*>(out) + (row * ld + col) * kSize;
    kept = k.matrix ? static_cast<char*>(k.matrix) + (row * k.ld + col) * kSize
                    : reinterpret_cast<char*>(k.packed.codes) + row * cols + col;
    exponent = k.packed.exponents + row * blocks(cols) + col / kBlock8;
  }
  __device__ __forceinline__ void down(int rows, int64_t ld, const Kept& k, int64_t cols) {
    y += rows * ld * kSize;
    kept += k.matrix ? rows * k.ld * kSize : rows * cols;
    exponent += rows * blocks(cols);
  }
};
template <int kType, int kHalves>
struct Targets {
  Target<kType> t0, t1;
  __device__ __forceinline__ void init(const End& e, int64_t row, int64_t col) {
    t0.init(e.y0, e.ld0, e.keep0, e.cols, row, col);
    if constexpr (kHalves == 2) t1.init(e.y1, e.ld1, e.keep1, e.cols, row, col);
  }
  __device__ __forceinline__ void down(const End& e, int rows) {
    t0.down(rows, e.ld0, e.keep0, e.cols);
    if constexpr (kHalves == 2) t1.down(rows, e.ld1, e.keep1, e.cols);
  }
};

// What the end of 8 columns from `col` adds to their sums, zeros where there is none.
__device__ __forceinline__ void load_bias(const float* bias, int64_t col, int64_t cols, float* b) {
  load_cols<8>(bias, col, POINTID_FP32, bias && col < cols ? cols - col : 0, b);
}
// the columns of a piece of 8 that exist, from `col` of `cols`
__device__ __forceinline__ int piece_cols(int64_t cols, int64_t col) {
  return cols - col < 8 ? (cols - col < 0 ? 0 : (int)(cols - col)) : 8;
}

// 8 values of a row (n exist, the rest are 0) as they stand in memory at p: read now, used
// later.
template <int kType>
struct Raw8 {
  static constexpr int kWords = kType == POINTID_FP32 ? 8 : 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const char* p, int n) {
    if (n >= 8) {
      __builtin_memcpy(w, p, sizeof(w));
      return;
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
    if (n <= 0) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i >= n) continue;
      if constexpr (kType == POINTID_FP32)
        w[i] = reinterpret_cast<const uint32_t*>(p)[i];
      else
        w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << (16 * (i % 2));
    }
  }
  __device__ __forceinline__ void values(float* v) const {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (kType == POINTID_FP32) {
        v[i] = __uint_as_float(w[i]);
      } else {
        v[2 * i] = from16((uint16_t)w[i], kType);
        v[2 * i + 1] = from16((uint16_t)(w[i] >> 16), kType);
      }
    }
  }
};
// The same of a checkpoint: codes at c, the block's exponent at x.
struct RawCodes {
  uint32_t w[2];
  uint32_t exponent;
  __device__ __forceinline__ void load(const uint8_t* c, const uint8_t* x, int n) {
    w[0] = w[1] = 0;
    exponent = 127;
    if (n <= 0) return;
    exponent = *x;
    if (n >= 8) {
      __builtin_memcpy(w, c, 8);
      return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) w[i / 4] |= (uint32_t)c[i] << (8 * (i % 4));
  }
  __device__ __forceinline__ void values(float* v) const {
    unpack8(w[0], (int)exponent - 127, v);
    unpack8(w[1], (int)exponent - 127, v + 4);
  }
};

// The residual of 8 columns, zeros where there is none.
template <int kType>
struct Residual : Raw8<kType> {
  static __device__ __forceinline__ const char* at(const End& e, int64_t row, int64_t col) {
    return static_cast<const char*>(e.residual) + (row * e.ld_residual + col) * (kType == POINTID_FP32 ? 4 : 2);
  }
  __device__ __forceinline__ void add_to(float* v) const {
    float r[8];
    this->values(r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += r[i];
  }
};

// The factor of kEndStore's sums.
template <int kType>
__device__ __forceinline__ float unscale_of(const End& e) {
  if constexpr (kType != POINTID_FP16) return 1.f;
  return e.unscale ? *e.unscale : 1.f;
}

// The end of 8 finished columns of a row (see End), of which the first n exist; v1 and b1:
// the second half's, with kHalves == 2; b0, b1: load_bias's; r: the residual's.  The 4 lanes
// of an aligned group hold 32 columns of one row, from a multiple of 32 on (the lane `first`
// the first of them), and all call it; `live` is false where the row or the columns do not
// exist.  unscale: unscale_of's.
template <int kType, int kHalves>
__device__ __forceinline__ void finish(const End& e, const Targets<kType, kHalves>& to, bool live, bool first, int n,
                                       float* v0, float* v1, const float* b0, const float* b1, const Residual<kType>& r, float unscale) {
  if (e.mode == kEndStore) {
    if (!live) return;
    if constexpr (kType == POINTID_FP16)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v0[i] *= unscale;
        if constexpr (kHalves == 2) v1[i] *= unscale;
      }
    store_cols<8>(to.t0.y, 0, kType, n, v0);
    if constexpr (kHalves == 2) store_cols<8>(to.t1.y, 0, kType, n, v1);
    return;
  }
  auto keep = [&](const Target<kType>& t, const Kept& k, const float* v) {
    if (k.matrix) {
      if (live) store_cols<8>(t.kept, 0, kType, n, v);
    } else if (k.packed.codes) {
      save_codes(reinterpret_cast<uint8_t*>(t.kept), t.exponent, live, first, n, v);
    }
  };
#pragma unroll
  for (int i = 0; i < 8; ++i) v0[i] += b0[i];
  keep(to.t0, e.keep0, v0);
  if constexpr (kHalves == 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v1[i] += b1[i];
    keep(to.t1, e.keep1, v1);
  }
  if (!live) return;
  activate8(e.act, v0);
  if constexpr (kHalves == 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v0[i] *= v1[i];
  } else {
    r.add_to(v0);
  }
  store_cols<8>(to.t0.y, 0, kType, n, v0);
}
// A checkpoint's 8 values of a row from column `col`, a multiple of 8.
__device__ __forceinline__ void load_codes(const Packed8& s, int64_t row, int64_t col, int64_t cols, float* v) {
  RawCodes r;
  r.load(s.codes + row * cols + col, s.exponents + row * ((cols + kBlock8 - 1) / kBlock8) + col / kBlock8,
         piece_cols(cols, col));
  r.values(v);
}

// Block `block` of the column sums, by kThreads threads: 32 of them a row of the partial sums
// in turn; added in order at the end.  sums: kThreads / 32 * 33 values.
template <int kThreads>
__device__ __forceinline__ void sum_columns(const SumsJobs& a, uint32_t block, float* sums) {
  constexpr int kSubs = kThreads / 32;
  const uint32_t strips = (uint32_t)((a.cols + 31) / 32);
  const int h = block >= strips;
  float* const out = a.out[h];
  if (!out) return;
  const int c = threadIdx.x % 32, sub = threadIdx.x / 32;
  const int64_t col = (int64_t)(block - h * strips) * 32 + c, pitch = a.halves * a.cols;
  const float* const part = a.part + h * a.cols + col;
  float t = 0.f;
  if (col < a.cols)
#pragma unroll 4
    for (int64_t b = sub; b < a.rows; b += kSubs) t += part[b * pitch];
  sums[sub * 33 + c] = t;
  __syncthreads();
  if (sub != 0 || col >= a.cols) return;
  float v = 0.f;
#pragma unroll
  for (int s = 0; s < kSubs; ++s) v += sums[s * 33 + c];
  out[col] = v;
}

// 8 columns of partial sums (fp32, rows padded to whole blocks of 32 columns)
__device__ __forceinline__ void store_partial(const End& e, int split, int half, bool live, int64_t row, int64_t col,
                                              const float* v) {
  if (!live || col >= e.part_ld) return;
  float4* p = reinterpret_cast<float4*>(e.part + (((int64_t)split * e.halves + half) * e.rows + row) * e.part_ld + col);
  p[0] = make_float4(v[0], v[1], v[2], v[3]);
  p[1] = make_float4(v[4], v[5], v[6], v[7]);
}

}  // namespace pointid
