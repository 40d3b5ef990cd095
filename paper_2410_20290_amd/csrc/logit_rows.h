// Rows of logits: a wave's tile of 1024 entries, and entries as words in the order
// "larger value, then lower index".
#pragma once

#include "common.h"

namespace sr {

constexpr int kLpTile = 1024;     // entries of a wave's tile: 16 per lane

__device__ __forceinline__ uint64_t entry_word(float v, int i) {
  uint32_t u = __float_as_uint(v);
  if ((u & 0x7FFFFFFFu) == 0u) u = 0u;   // -0 == +0
  u = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return ((uint64_t)u << 32) | (uint32_t)~i;
}
__device__ __forceinline__ float word_value(uint64_t w) {
  const uint32_t u = (uint32_t)(w >> 32);
  return __uint_as_float((u & 0x80000000u) ? (u & 0x7FFFFFFFu) : ~u);
}
__device__ __forceinline__ int word_index(uint64_t w) { return (int)~(uint32_t)w; }


// A tile's 16 entries of this lane, and their indices: aligned rows take 16
// bytes a load, others an element; past the end: NaN (counts as -inf).
template <typename T, bool VEC>
struct Tile {
  static constexpr int N = 16 / sizeof(T);   // entries of a 16-byte load
  __device__ __forceinline__ static int index(int base, int e, int lane) {
    return VEC ? base + (e / N) * 64 * N + N * lane + e % N : base + 64 * e + lane;
  }
  __device__ __forceinline__ static void load(const T* __restrict__ x, int base, int end, int lane, float (&v)[16]) {
    if (VEC && base + kLpTile <= end) {
#pragma unroll
      for (int q = 0; q < 16 / N; ++q) Vec16<T>::load(x + base + q * 64 * N + N * lane, v + q * N);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int i = index(base, e, lane);
        v[e] = i < end ? to_f32<T>(x[i]) : __uint_as_float(0x7FC00000u);
      }
    }
  }
};

}  // namespace sr
