// The 8-bit cache's numbers: e4m3 values beside a power-of-two scale for each 16 tokens of a KV position.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace twist {

constexpr int kScaleTokens = 16;          // tokens that share a scale
constexpr int kScaleLow = -110, kScaleHigh = 119;

// The smallest power of two 2^e, kScaleLow <= e <= kScaleHigh, whose 448-fold (the largest e4m3 number) is not below `top` >= 0.
__device__ inline float scale_for(float top) {
  const uint32_t u = __float_as_uint(top);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);          // 448 = 1.75 * 2^8
  return __uint_as_float((uint32_t)(min(max(e, kScaleLow), kScaleHigh) + 127) << 23);
}
// The power of two in that range which counts for a block's old scale: the next one from it on; what is not positive counts for nothing.
__device__ inline float scale_above(float old) {
  const uint32_t u = __float_as_uint(old);
  const int e = old > 0.f ? (int)(u >> 23) - 127 + ((u & 0x7fffffu) != 0) : kScaleLow;
  return __uint_as_float((uint32_t)(min(max(e, kScaleLow), kScaleHigh) + 127) << 23);
}
// 1 / scale for a power of two in that range (exact).
__device__ inline float inverse_scale(float scale) { return __uint_as_float((254u << 23) - __float_as_uint(scale)); }

// Two values as e4m3 numbers, to nearest even, saturating; the first in the low byte.  What is not finite becomes NaN.
__device__ inline uint32_t narrow2(float lo, float hi) {
  lo = fabsf(lo) < INFINITY ? lo : __int_as_float(0x7fffffff);
  hi = fabsf(hi) < INFINITY ? hi : __int_as_float(0x7fffffff);
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// The same for values that are finite.
__device__ inline uint32_t narrow4_finite(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
      : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
__device__ inline uint32_t narrow4(float a, float b, float c, float d) { return narrow2(a, b) | (narrow2(c, d) << 16); }

// Four e4m3 numbers (exact).
__device__ inline void widen4(float (&a)[4], uint32_t v) {
  uint32_t lo, hi;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(v));
  const float2 x = __half22float2(*reinterpret_cast<__half2*>(&lo)), y = __half22float2(*reinterpret_cast<__half2*>(&hi));
  a[0] = x.x; a[1] = x.y; a[2] = y.x; a[3] = y.y;
}

}  // namespace twist
