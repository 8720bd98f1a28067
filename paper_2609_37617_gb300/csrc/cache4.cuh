// cache4.cuh -- the format of a cache in 4 bits (include/as2d.h, as2d_cache4): 16
// consecutive dims share a scale s and hold whole numbers c in -7 .. 7, for s c.
//
// Why this one.  s has four significant bits and c three, so that s c is exact in
// bf16 and in 16-bit floats: what attends to the cache multiplies exact values, and
// a decoded value costs one fused multiply-add of two halves.  A scale byte is the
// upper byte of a non-negative 16-bit float (less its sign), decoded by a shift, with a
// range of 2^-17 to 896 that needs no further factor.  16 dims to a scale: 4.5 bits
// a value; uniform steps of a seventh of the largest are off by 8.5 % (root mean square)
// of N(0, 1) values, the eight magnitudes of a 4-bit float by 9.8 %.
#pragma once

#include <cuda_fp16.h>

#include "ops.h"

namespace as2d {

constexpr float kMaxScale4 = 896.f;  // 72 of them fit a 16-bit float (scale_shift)

__device__ __forceinline__ uint8_t scale_byte(float s) { return (uint8_t)(__half_as_ushort(__float2half_rn(s)) >> 7); }

// ---- coding ---------------------------------------------------------------------
//
// Exact values of 8 significant bits (bf16) need no division: x / s with s of four bits,
// and a largest magnitude over 7 in steps of scales, are on the border of two whole numbers or
// at least 2^-10 from it where they are over 0.4, so that a product with the reciprocal (off by 2^-20), rounded
// to 2^-12, is on the border just where they are.  (on_grid(x, f): x f so rounded, for |x f| <= 16.)
__device__ __forceinline__ float on_grid(float x, float f) { return fmaf(x, f, 2304.f) - 2304.f; }

__device__ __forceinline__ float reciprocal(float s) { return s > 0.f ? __fdividef(1.f, s) : 0.f; }

// The scale of exact bf16 values whose largest magnitude is `most`.
__device__ __forceinline__ float exact_scale(float most) {
  const float t = most * (1.f / 7.f);
  const int e = min(max((int)(__float_as_uint(t) >> 23), 127 - 14), 127 + 9);
  const float steps = fminf(most, 7168.f) * __uint_as_float((uint32_t)(2 * 127 + 3 - e) << 23);  // of 1/7
  return fminf(rintf(fminf(on_grid(steps, 1.f / 7.f), 16.f)) * __uint_as_float((uint32_t)(e - 3) << 23), kMaxScale4);
}

// The code of x / s, s = 1 / inv, as the lowest bits of the result, for exact values: the product on
// the grid, then rounded to a whole number by an addition whose sum's last place is 1.  With
// |x inv| < 7.5 (scales of 2^-14 and more that are not capped); clamped: for all.
__device__ __forceinline__ uint32_t code_bits(float x, float inv) {
  return __float_as_uint(fmaf(x, inv, 2304.f) + (12582912.f + 8.f - 2304.f));
}
__device__ __forceinline__ uint32_t code_bits_clamped(float x, float inv) {
  return __float_as_uint(fminf(fmaxf(on_grid(x, inv), -7.f), 7.f) + (12582912.f + 8.f));
}
// The same of values that are not exact, rounded where they are.
__device__ __forceinline__ uint32_t code_bits_near(float q) {
  return __float_as_uint(fminf(fmaxf(q, -7.f), 7.f) + (12582912.f + 8.f));
}
// The word of 8 codes.
__device__ __forceinline__ uint32_t code_word(const uint32_t (&c)[8]) {
  uint32_t w = 0;
#pragma unroll
  for (int e = 3; e >= 0; --e) w = w * 16 + __byte_perm(c[2 * e], c[2 * e + 1], 0x5410);
  return w;
}

// ---- decoding -------------------------------------------------------------------
//
// A code n over the significand of a half whose exponent gives its place the value 1: 64 + n in bits
// 4 .. 7, of which one fused multiply-add makes (64 + n) s - 72 s = (n - 8) s; and 1024 + n in bits 0
// .. 3, less 1032 first (1032 s is no half).  So a word's eight codes take one shift and four
// logic operations, the rest runs where products do.  All steps are exact.

// s of two scale bytes (16 bits apart), and -72 s.
__device__ __forceinline__ __half2 scale_pair(uint32_t bytes) {
  const uint32_t b = bytes * 128u;
  return __hmin2(*reinterpret_cast<const __half2*>(&b), __float2half2_rn(kMaxScale4));
}
__device__ __forceinline__ __half2 scale_shift(__half2 s) { return __hmul2(s, __float2half2_rn(-72.f)); }

// The four pairs of codes in a word (each 16 bits apart): pair e is at bits 4e.
__device__ __forceinline__ void decode_word(uint32_t w, __half2 s, __half2 shift, __half2 (&v)[4]) {
#pragma unroll
  for (int e = 0; e < 4; e += 2) {
    const uint32_t u = e ? w >> 8 : w;
    const uint32_t x = (u & 0x000F000Fu) | 0x64006400u, y = (u & 0x00F000F0u) | 0x54005400u;
    v[e] = __hmul2(__hadd2(*reinterpret_cast<const __half2*>(&x), __float2half2_rn(-1032.f)), s);
    v[e + 1] = __hfma2(*reinterpret_cast<const __half2*>(&y), s, shift);
  }
}

}  // namespace as2d
