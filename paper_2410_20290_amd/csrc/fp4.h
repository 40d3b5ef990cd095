// The 4-bit cache format: groups of 32 dimensions, each e2m1 (sign, 0 0.5 1 1.5 2
// 3 4 6) times the group's 2^(b - 127).  A page's codes of one KV head come first,
// [page_tokens][head_dim / 2] bytes, then the bytes b [page_tokens][head_dim / 32].
#pragma once

#include "common.h"
#include "paged.h"

namespace sr {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Byte offset of a page's block of one KV head, and of a slot's codes and scale
// bytes in it.
SR_HD int64_t fp4_block(int pg, int n_kv_heads, int h, int shift, int head_dim) {
  return (((int64_t)pg * n_kv_heads + h) << shift) * (head_dim * 17 / 32);
}
SR_HD int fp4_codes(int slot, int head_dim) { return slot * (head_dim / 2); }
SR_HD int fp4_scales(int slot, int shift, int head_dim) {
  return (head_dim / 2 << shift) + slot * (head_dim / 32);
}

// Writing.  A magnitude travels as the upper half of a double's bits with a bit
// for what the lower half holds: all borders between codes have three significant
// bits, so every comparison with one is exact.
__device__ __forceinline__ uint32_t fp4_mag(double x) {
  const uint64_t u = (uint64_t)__double_as_longlong(x);
  return ((uint32_t)(u >> 32) & 0x7FFFFFFFu) | ((uint32_t)u != 0u ? 1u : 0u);
}
// The scale byte of a group whose largest magnitude is `top`.
__device__ __forceinline__ int fp4_scale_byte(uint32_t top) {
  if (top >= 0x7FF00000u) return 255;
  const int e = (int)(top >> 20) - 1023 + ((top & 0xFFFFFu) >= 0xC0000u ? 1 : 0);   // (1.75 up counts as 2)
  return imax(2, imin(252, e - 2 + 127));
}
__device__ __forceinline__ uint32_t fp4_code(double x, int byte) {
  if (byte == 255) return 0u;
  const int s = (int)fp4_mag(x) - (byte - 127) * (1 << 20);
  const uint32_t c = (s > 0x3FD00000) + (s >= 0x3FE80000) + (s > 0x3FF40000) + (s >= 0x3FFC0000) +
                     (s > 0x40040000) + (s >= 0x400C0000) + (s > 0x40140000);
  return c | ((uint32_t)((uint64_t)__double_as_longlong(x) >> 63) << 3);
}

// Reading.  The scale as the fp32 whose exponent the conversions take; 255 is NaN.
__device__ __forceinline__ float fp4_scale(uint32_t byte) {
  return __uint_as_float(byte == 255u ? 0x7FC00000u : byte << 23);
}
__device__ __forceinline__ float fp4_value(uint32_t code, float scale) {
  const uint32_t m = code & 7u;
  // 0 and 0.5, then (2 + low bit) 2^(m / 2 - 2)
  const float v = m < 2u ? 0.5f * (float)m : __uint_as_float(((126u + (m >> 1)) << 23) | ((m & 1u) << 22));
  return ((code & 8u) ? -v : v) * scale;
}

// Eight codes (a word, the lowest first) times a scale, as bf16.
__device__ __forceinline__ bf16x8 fp4_to_bf16(uint32_t w, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

}  // namespace sr
