// Loads and stores of 8 values of a row that need not stay in the caches.
#pragma once

#include "internal.h"
#include "layers_end.h"

namespace pointid {

// Whether a call that reads and writes so many matrices does not keep them in the 256 MB of the
// last-level cache for whatever comes next: then loads and stores without a place in the caches
// are faster, below slower, and of fp32, whose 8 values are two accesses a lane, never faster.
// Plain and passing, us: bf16 dropout of 2048 x 8192 with a residual (101 MB) 18.6 and 20.5, 4096 x
// 8192 (201 MB) 36.4 and 37.6, 8192 x 8192 (403 MB) 75 and 68, 16384 x 8192 (805 MB) 148 and 132; a
// joint's gradients of 8192 x 4096 (403 MB) 89 and 82, 16384 x 4096 157 and 148; the joint of 8192 x
// 4096 (268 MB) 52 and 58, of 16384 x 4096 (537 MB) 107 and 103; fp32 1693 x 32003 logits' gradient
// (433 MB) 84 and 94.
inline bool passes_cache(int dtype, int64_t rows, int64_t cols, int matrices) {
  return dtype != POINTID_FP32 && 2 * rows * cols * matrices >= int64_t(384) << 20;
}

typedef uint32_t Words4 __attribute__((ext_vector_type(4), aligned(2)));

template <int kType>
struct Passing {
  // raw.load(p, n) and store_cols, where `passing` without a place in the caches
  static __device__ __forceinline__ void load(Raw8<kType>* raw, const char* p, int n, bool passing) {
    if constexpr (kType != POINTID_FP32) {
      if (passing && n >= 8) {
        const Words4 w = __builtin_nontemporal_load(reinterpret_cast<const Words4*>(p));
        __builtin_memcpy(raw->w, &w, 16);
        return;
      }
    }
    raw->load(p, n);
  }
  static __device__ __forceinline__ void store(char* p, int n, const float (&v)[8], bool passing) {
    if (n >= 8) {
      if constexpr (kType == POINTID_FP32) {
        __builtin_memcpy(p, v, 32);
      } else {
        const Words4 w = {pack16(v[0], v[1], kType), pack16(v[2], v[3], kType), pack16(v[4], v[5], kType),
                          pack16(v[6], v[7], kType)};
        if (passing)
          __builtin_nontemporal_store(w, reinterpret_cast<Words4*>(p));
        else
          __builtin_memcpy(p, &w, 16);
      }
      return;
    }
    // (not the eighth: the compiler would take its store out of both cases, and a whole piece's 32
    // bytes would be three stores; fp32 1693 x 32003 logits' gradient 94 us for 84)
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) store_any(p, i, v[i], kType);
  }
};

}  // namespace pointid
