// The integer weights by which tokens are drawn, and sums of them across lanes.
// Include it only where floating-point contraction is off: every step is a
// separately rounded float32 operation.
#pragma once

#include "common.h"

#pragma clang fp contract(off)

namespace sr {

// trunc(exp_sr((l - m) / T) * 2^32) as a saturating 32-bit word: 2^32 itself
// (exp_sr = 1) comes back as 0xFFFFFFFF, which no smaller float truncates to.
// The same rounded steps in fewer instructions:
//  - n = rint(z log2 e) by adding 1.5 * 2^23 + 32 (an even offset, so ties
//    round alike); the low bits of the sum are n + 32, added to the exponent
//    of the polynomial, which is the exact scaling by 2^n 2^32;
//  - arguments below -24, -inf and NaN are clamped to -25, where the weight
//    truncates to 0 like that of every argument below -22.2.
__device__ __forceinline__ uint32_t weight32(float l, float m, float inv_t) {
  const float kLog2e = __uint_as_float(0x3FB8AA3Bu);
  const float kLn2Hi = __uint_as_float(0x3F317200u);
  const float kLn2Lo = __uint_as_float(0x35BFBE8Eu);
  const float c2 = 0.5f, c3 = __uint_as_float(0x3E2AAAABu), c4 = __uint_as_float(0x3D2AAAABu),
              c5 = __uint_as_float(0x3C088889u), c6 = __uint_as_float(0x3AB60B61u),
              c7 = __uint_as_float(0x39500D01u);
  const float kRound = 12582912.0f + 32.0f;
  const float z = fmaxf(__fmul_rn(__fsub_rn(l, m), inv_t), -25.0f);
  const float t = __fadd_rn(__fmul_rn(z, kLog2e), kRound);
  const float n = __fsub_rn(t, kRound);
  float r = __fsub_rn(z, __fmul_rn(n, kLn2Hi));
  r = __fsub_rn(r, __fmul_rn(n, kLn2Lo));
  float p = c7;
  p = __fadd_rn(__fmul_rn(p, r), c6);
  p = __fadd_rn(__fmul_rn(p, r), c5);
  p = __fadd_rn(__fmul_rn(p, r), c4);
  p = __fadd_rn(__fmul_rn(p, r), c3);
  p = __fadd_rn(__fmul_rn(p, r), c2);
  p = __fadd_rn(__fmul_rn(p, r), 1.0f);
  p = __fadd_rn(__fmul_rn(p, r), 1.0f);
  const float x = __uint_as_float(__float_as_uint(p) + (__float_as_uint(t) << 23));
  uint32_t w;
  asm("v_cvt_u32_f32 %0, %1" : "=v"(w) : "v"(x));
  return w;
}

__device__ __forceinline__ uint64_t weight_of(float l, float m, float inv_t) {
  const uint32_t w = weight32(l, m, inv_t);
  return (uint64_t)w + (w == 0xFFFFFFFFu ? 1u : 0u);
}

__device__ __forceinline__ uint64_t shfl_xor_u64(uint64_t v, int o) {
  uint32_t lo = (uint32_t)v, hi = (uint32_t)(v >> 32);
  lo = __shfl_xor(lo, o, 64);
  hi = __shfl_xor(hi, o, 64);
  return ((uint64_t)hi << 32) | lo;
}
__device__ __forceinline__ uint64_t shfl_up_u64(uint64_t v, int o) {
  uint32_t lo = (uint32_t)v, hi = (uint32_t)(v >> 32);
  lo = __shfl_up(lo, o, 64);
  hi = __shfl_up(hi, o, 64);
  return ((uint64_t)hi << 32) | lo;
}

}  // namespace sr
