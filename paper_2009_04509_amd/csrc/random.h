// Random bits from a counter, and the dropout made of them.
//
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3,
// SC 2011): 10 rounds of two 32 x 32 -> 64 bit products turn a counter of four words and a
// key of two into four random words.  Element (row, col) has 16 of the 128 bits of the counter
// (col / 8, row, offset's lower word, its upper word) under the key `seed`: word (col % 8) / 2,
// its lower half for even columns.  It depends on nothing else, so that a gradient (or a second
// forward pass) makes the mask again instead of reading one.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "internal.h"

namespace pointid {

struct Drop {
  uint32_t threshold;          // kept: 16 random bits of at least this; 0: no dropout
  float scale;                 // 65536 / (65536 - threshold), one over the share that is kept; 0 of none
  uint64_t seed, offset;
  const uint64_t* step;        // device memory, added to the offset, or nullptr
};

// A launch's key and the counter's constant words.
struct DropKey {
  uint32_t k0, k1, c2, c3;
  __device__ __forceinline__ explicit DropKey(const Drop& d) {
    const uint64_t at = d.offset + (d.step ? *d.step : 0);
    k0 = (uint32_t)d.seed, k1 = (uint32_t)(d.seed >> 32);
    c2 = (uint32_t)at, c3 = (uint32_t)(at >> 32);
  }
};

__device__ __forceinline__ void philox(const DropKey& key, uint32_t c0, uint32_t c1, uint32_t (&w)[4]) {
  uint32_t c2 = key.c2, c3 = key.c3, k0 = key.k0, k1 = key.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)b;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  w[0] = c0, w[1] = c1, w[2] = c2, w[3] = c3;
}

// v of columns col .. col + 7 (col a multiple of 8) through the dropout.  What is dropped is 0
// whatever it was, an infinity or NaN too; where `with` is given, its values there are 0 as well.
__device__ __forceinline__ void drop8(const Drop& d, const DropKey& key, int64_t row, int64_t col, float (&v)[8],
                                      float (*with)[8] = nullptr) {
  uint32_t w[4];
  philox(key, (uint32_t)(col / 8), (uint32_t)row, w);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t bits = i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu;
    const bool kept = bits >= d.threshold;
    v[i] = kept ? v[i] * d.scale : 0.f;
    if (with) (*with)[i] = kept ? (*with)[i] : 0.f;
  }
}

}  // namespace pointid
