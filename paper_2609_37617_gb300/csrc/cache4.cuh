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

// The scale nearest to t >= 0 (ties to even); units: t in steps of the scales around it.
template <typename T>
__device__ __forceinline__ float scale_of(T t, T& units) {
  // steps of 2^(e - 3), e the exponent of t, at least that of the smallest normal scale
  // (t rounded up to a power of two gives the same scale)
  const int e = min(max((int)(__float_as_uint((float)t) >> 23), 127 - 14), 127 + 9);
  units = t * (T)__uint_as_float((uint32_t)(2 * 127 + 3 - e) << 23);
  const float r = fminf((float)rint(units), 16.f);  // (16: the next exponent's first)
  return fminf(r * __uint_as_float((uint32_t)(e - 3) << 23), kMaxScale4);
}
__device__ __forceinline__ uint8_t scale_byte(float s) { return (uint8_t)(__half_as_ushort(__float2half_rn(s)) >> 7); }

// The codes of 8 values in a word.
__device__ __forceinline__ uint32_t code_word(const int (&c)[8]) {
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    w |= (uint32_t)(c[2 * e] + 8) << (4 * e) | (uint32_t)(c[2 * e + 1] + 8) << (16 + 4 * e);
  return w;
}

// c = x / s to the nearest, ties to even.  The quotient of 8 significant bits by four is
// never so near to a border that its rounding to 32 bits would cross it.
__device__ __forceinline__ int code_of(float x, float s) {
  return s > 0.f ? (int)rintf(fminf(fmaxf(__fdiv_rn(x, s), -7.f), 7.f)) : 0;
}

// ---- decoding -------------------------------------------------------------------
//
// (64 + n) s - 72 s = (n - 8) s in one fused multiply-add of two halves: the
// significand of 64 + n holds the code n in bits 4 .. 7.

// s of a scale byte, twice, and -72 s.
__device__ __forceinline__ __half2 scale_pair(uint32_t bytes) {  // two bytes, 16 bits apart
  const uint32_t b = (bytes & 0x00FF00FFu) << 7;
  return __hmin2(*reinterpret_cast<const __half2*>(&b), __float2half2_rn(kMaxScale4));
}
__device__ __forceinline__ __half2 scale_shift(__half2 s) { return __hmul2(s, __float2half2_rn(-72.f)); }

// The four pairs of codes in a word (each 16 bits apart): pair e is at bits 4e.
__device__ __forceinline__ void decode_word(uint32_t w, __half2 s, __half2 shift, __half2 (&v)[4]) {
  const uint32_t m = 0x00F000F0u, one = 0x54005400u;
  const uint32_t x[4] = {((w << 4) & m) | one, (w & m) | one, ((w >> 4) & m) | one, ((w >> 8) & m) | one};
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = __hfma2(*reinterpret_cast<const __half2*>(&x[e]), s, shift);
}

}  // namespace as2d
