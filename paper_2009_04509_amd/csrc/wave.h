// Sums and maxima over lanes by DPP and the lane swaps of gfx950, without shared memory, every
// lane with the result; the order is always the same.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace pointid {

// Of 4-byte values: those of the lanes that a DPP control gives.
template <int kControl, class T>
__device__ __forceinline__ T dpp(T v) {
  return __builtin_bit_cast(T, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), kControl, 0xF, 0xF, true));
}
constexpr int kPairs = 0xB1, kQuads = 0x4E, kQuadMirror = 0x1B, kHalfMirror = 0x141, kRowMirror = 0x140, kRowTurn8 = 0x128;
// The value and that of the lane 16 (32) away, the one of the even row (lower half) first.
template <class T>
__device__ __forceinline__ void rows_swapped(T v, T* even, T* odd) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v);
  auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  *even = __builtin_bit_cast(T, (uint32_t)r[0]);
  *odd = __builtin_bit_cast(T, (uint32_t)r[1]);
}
template <class T>
__device__ __forceinline__ void halves_swapped(T v, T* low, T* high) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v);
  auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  *low = __builtin_bit_cast(T, (uint32_t)r[0]);
  *high = __builtin_bit_cast(T, (uint32_t)r[1]);
}
// f over aligned groups of kLanes lanes (a power of two): pairs, quads, mirrored halves and rows
// of 16, rows, halves
template <int kLanes, class T, class F>
__device__ __forceinline__ T over_lanes(T v, F&& f) {
  T a, b;
  if constexpr (kLanes >= 2) v = f(v, dpp<kPairs>(v));
  if constexpr (kLanes >= 4) v = f(v, dpp<kQuads>(v));
  if constexpr (kLanes >= 8) v = f(v, dpp<kHalfMirror>(v));
  if constexpr (kLanes >= 16) v = f(v, dpp<kRowMirror>(v));
  if constexpr (kLanes >= 32) {
    rows_swapped(v, &a, &b);
    v = f(a, b);
  }
  if constexpr (kLanes == 64) {
    halves_swapped(v, &a, &b);
    v = f(a, b);
  }
  return v;
}
template <int kLanes>
__device__ __forceinline__ float lanes_sum(float v) {
  return over_lanes<kLanes>(v, [](float a, float b) { return a + b; });
}
template <int kLanes>
__device__ __forceinline__ float lanes_max(float v) {
  return over_lanes<kLanes>(v, [](float a, float b) { return fmaxf(a, b); });
}
// The value of lane ^ kX, kX a power of two or 63.
template <int kX>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
  if constexpr (kX == 1) return dpp<kPairs>(v);
  if constexpr (kX == 2) return dpp<kQuads>(v);
  if constexpr (kX == 4) return dpp<kQuadMirror>(dpp<kHalfMirror>(v));
  if constexpr (kX == 8) return dpp<kRowTurn8>(v);
  uint32_t a, b;
  if constexpr (kX == 16) {
    rows_swapped(v, &a, &b);
    return threadIdx.x & 16 ? a : b;
  }
  if constexpr (kX == 32) {
    halves_swapped(v, &a, &b);
    return threadIdx.x & 32 ? a : b;
  }
  return lane_xor<32>(lane_xor<16>(dpp<kRowMirror>(v)));
}

}  // namespace pointid
