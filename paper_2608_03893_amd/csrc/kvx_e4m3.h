// OCP e4m3 helpers of the 8-bit pool (device code only).
#pragma once

#include "kvx_bf16.h"

namespace kvx {

constexpr int kScaleExpMin = -118;   // least exponent of a page's scale

// The smallest power of two s, at least 2^kScaleExpMin, with amax <= 448 s, for finite
// amax >= 0: with amax = m 2^e, 1 <= m < 2, and 448 = 1.75 * 2^8, s = 2^(e - 8), or
// twice that when m > 1.75.  Exact: it only looks at the bits.
__device__ __forceinline__ float pow2_scale(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __uint_as_float((uint32_t)((e > kScaleExpMin ? e : kScaleExpMin) + 127) << 23);
}

// |x| where x is finite, else 0 (what a page's scale counts).
__device__ __forceinline__ float finite_abs(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return u < 0x7f800000u ? __uint_as_float(u) : 0.0f;
}

// Four values times r as e4m3 codes, nearest even, |x r| <= 448 for finite x.  Infinities
// become NaN (x + 0 x), which e4m3 has, so that they stay visible.
__device__ __forceinline__ uint32_t to_e4m3x4(float x0, float x1, float x2, float x3, float r) {
  x0 = __builtin_fmaf(x0, 0.0f, x0) * r;
  x1 = __builtin_fmaf(x1, 0.0f, x1) * r;
  x2 = __builtin_fmaf(x2, 0.0f, x2) * r;
  x3 = __builtin_fmaf(x3, 0.0f, x3) * r;
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, w, true);
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

constexpr uint32_t kNan4 = 0x7f7f7f7fu;   // four NaN codes

// The top bit of each byte that is NaN (all ones but the sign).
__device__ __forceinline__ uint32_t e4m3_nan(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// Code i (0 .. 3) of a word, exactly.
template <int I>
__device__ __forceinline__ float from_e4m3(uint32_t w) { return __builtin_amdgcn_cvt_f32_fp8((int)w, I); }

}  // namespace kvx
