// q4.cuh -- numbers in 4 bits: groups of 16 components that share a scale of
// 8 bits (4 of exponent, 3 of fraction); a code has a sign, 2 bits of
// exponent and 1 of fraction: 0, .5, 1, 1.5, 2, 3, 4, 6.
#pragma once
#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include <cstdint>

namespace simsd {

constexpr int kQ4Group = 16;

// A group's scale for the largest magnitude `top` of x / unit: a sixth of it,
// so that the largest component falls on 6, to nearest (at most 448, NaN for
// NaN); never 0, so that x / scale is defined.
__device__ __forceinline__ uint32_t q4_scale(float top) {
  // top / 6 correctly rounded: the product with fl(1 / 6) and one step of
  // correction by its residual (Markstein 1990).  The product alone puts some
  // numbers next below a border between two scales on it.  (An infinity, and
  // only that, has no residual.)
  float y = top * (1.f / 6.f);
  const float z = fmaf(fmaf(-6.f, y, top), 1.f / 6.f, y);
  if (top < INFINITY) y = z;
  const uint32_t s = __nv_cvt_float_to_fp8(y, __NV_SATFINITE, __NV_E4M3);
  return s == 0 ? 1u : s;
}
__device__ __forceinline__ float q4_scale_value(uint32_t s) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<__nv_fp8_storage_t>(s), __NV_E4M3)));
}
// The codes of two quotients, the first in the low half: to nearest, ties to
// even, at most 6.
__device__ __forceinline__ uint32_t q4_codes(float a, float b) {
  return __nv_cvt_float2_to_fp4x2(make_float2(a, b), __NV_E2M1, cudaRoundNearest);
}

// The two codes of byte `i` of w as fp16 (low half of the byte first).
template <int i>
__device__ __forceinline__ uint32_t q4_pair(uint32_t w) {
  uint32_t h;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "mov.b32 {b0, b1, b2, b3}, %1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b%2;\n\t}"
      : "=r"(h)
      : "r"(w), "n"(i));
  return h;
}
// Two scales (the low 16 bits of s) as fp16.
__device__ __forceinline__ uint32_t q4_scale_pair(uint32_t s) {
  uint32_t h;
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "mov.b32 {lo, hi}, %1;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, lo;\n\t}"
      : "=r"(h)
      : "r"(s));
  return h;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

}  // namespace simsd
