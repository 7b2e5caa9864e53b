// Codes of 4 bits (OCP e2m1: sign, 0 0.5 1 1.5 2 3 4 6) in groups of 32 with one power of two each, as the byte e + 127: keys and values in the pages
// (DP_KV_FP4) and weights (dp_linear_fp4).  The least e in [-100, 125] that brings every finite |x| of the group to 7 = 1.75 * 2^2 or below: 6 to 7 round to
// the largest code, off by at most half the step below it, and the range of codes is used whole.  The product with 2^-e is exact, so the code is
// the only rounding (x * 2^-e below 2^-126 is far below half a code).  Beyond 7 * 2^125 the conversion saturates, which only values above 1.75 * 2^127 reach:
// the next factor's 4 would stand for 2^128.
#pragma once
#include "common.h"

constexpr int FP4_GROUP = 32;
constexpr uint32_t FP4_NAN = 255;         // a group's byte: a value of it was not finite, and all read back as NaN

__device__ __forceinline__ int fp4_exponent(float amax) {          // amax finite
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 127 - 2 + ((b & 0x7fffffu) > 0x600000u);
  return e < -100 ? -100 : e > 125 ? 125 : e;
}
// the group's byte from its largest |x|, infinity if one is not finite
__device__ __forceinline__ uint32_t fp4_byte(float amax) { return amax < INFINITY ? (uint32_t)(fp4_exponent(amax) + 127) : FP4_NAN; }
// 2^-e, and 0 for a group that reads back as NaN: its codes are 0
__device__ __forceinline__ float fp4_inverse(uint32_t byte) { return byte == FP4_NAN ? 0.f : __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ float fp4_size(float x) { return fabsf(x) < INFINITY ? fabsf(x) : INFINITY; }
// The conversions round to nearest, ties to even, and saturate.  What is not finite is 0: its group is NaN by its byte.
__device__ __forceinline__ float fp4_scaled(float x, float inv) { return inv == 0.f ? 0.f : x * inv; }
__device__ __forceinline__ uint32_t to_fp4x4(float a, float b, float c, float d, float inv) {
  const uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, fp4_scaled(a, inv), fp4_scaled(b, inv), 1.f, 0);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, fp4_scaled(c, inv), fp4_scaled(d, inv), 1.f, 1);
}
// eight codes times the factor, packed bf16, four of them in fp32: exact.  The factor is handed over as the byte in a float's exponent, of which the
// conversion takes the 255 for NaN as well.
__device__ __forceinline__ uint4 fp4x8_to_bf16(uint32_t w, float scale) {
  auto h = [scale, w](auto at) __attribute__((always_inline)) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, decltype(at)::value));
  };
  return make_uint4(h(std::integral_constant<int, 0>{}), h(std::integral_constant<int, 1>{}), h(std::integral_constant<int, 2>{}), h(std::integral_constant<int, 3>{}));
}
__device__ __forceinline__ float4 fp4x4_to_f32(uint32_t w, float scale) {
  const f32_pair_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  return make_float4(a[0], a[1], b[0], b[1]);
}
