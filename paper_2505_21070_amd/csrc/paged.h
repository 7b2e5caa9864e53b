// What the kernels around the paged key/value cache share: where a token's head lies in the pages, codes of 8 bits, and the
// checks of rows and caches at the C entries.
#pragma once
#include "../../include/dualparal.h"
#include <stdio.h>

#include "common.h"

int dp_set_error(int code, const char* msg);   // defined next to dp_last_error

// DP_KV_FP8: a row of values x is held as codes e4m3(x * 2^-e) and the byte e + 127, with the least e >= -100 that brings every finite
// |x| to 448 = 1.75 * 2^8 or below.  Both products with a power of two are exact (x * 2^-e below e4m3's range rounds once, in the
// conversion), so the code is the only rounding.  The largest e is 120, where the code 256 would stand for 2^128, which neither fp32 nor bf16
// holds: values are bounded by 240 * 2^120 before the product (half a step off at most, as any code is; only rows with e = 120 reach the bound).
__device__ __forceinline__ int fp8_exponent(float amax) {          // amax finite
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u);
  return e < -100 ? -100 : e;
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127
// four values to four codes; what is not finite becomes NaN.  The bound costs nothing that can be measured: 40 + 40 heads of 6240 tokens into codes and back 80.1 us with it and without.
__device__ __forceinline__ uint32_t to_fp8x4(float a, float b, float c, float d, float inv) {
  auto f = [inv](float x) __attribute__((always_inline)) {
    return fabsf(x) < INFINITY ? __builtin_amdgcn_fmed3f(x, -0x1.ep127f, 0x1.ep127f) * inv : __uint_as_float(0x7fc00000u);
  };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(f(a), f(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f(c), f(d), w, true);
}
// eight codes times 2^e as packed bf16: exact (the conversion takes the factor's exponent)
__device__ __forceinline__ uint4 fp8x8_to_bf16(uint2 c, float scale) {
  auto h = [scale](uint32_t w, auto hi_) __attribute__((always_inline)) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, decltype(hi_)::value));
  };
  return make_uint4(h(c.x, std::false_type{}), h(c.x, std::true_type{}), h(c.y, std::false_type{}), h(c.y, std::true_type{}));
}
__device__ __forceinline__ float4 fp8x4_to_f32(uint32_t w, float scale) {
  const f32_pair_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
  return make_float4(a[0], a[1], b[0], b[1]);
}

// ---- host: checks at the C entries; each returns null, or why not
inline const char* why_not_head(int32_t heads, int32_t head_dim, int32_t dtype) {
  if (heads < 1 || heads > 1024) return "heads must be in [1, 1024]";
  if (head_dim != 64 && head_dim != 128) return "head_dim must be 64 or 128";
  if (dtype != DP_F32 && dtype != DP_BF16) return "dtype must be DP_F32 or DP_BF16";
  return nullptr;
}
inline const char* why_not_cache(const dp_kv_cache* c) {
  if (!c) return "null pointer";
  if (const char* why = why_not_head(c->kv_heads, c->head_dim, c->dtype)) return why;
  if (c->format != DP_KV_PLAIN && c->format != DP_KV_FP8) return "the cache's format must be DP_KV_PLAIN or DP_KV_FP8";
  if (c->page_tokens < 16 || c->page_tokens > 65536 || (c->page_tokens & (c->page_tokens - 1))) return "page_tokens must be a power of two in [16, 65536]";
  if (c->n_pages < 1 || (int64_t)c->n_pages * c->page_tokens > 0x7fffffff) return "n_pages * page_tokens must be in [1, 2^31 - 1]";
  if (!c->data || (c->format == DP_KV_FP8 && !c->scales)) return "null pointer";
  if ((uintptr_t)c->data & 15) return "the cache must be 16-byte aligned";
  return nullptr;
}
// rows of [n_tokens, heads, head_dim], n_tokens >= 1
inline const char* why_not_rows(const dp_rows* r, int64_t n_tokens, int32_t heads, int32_t head_dim, int32_t dtype, bool written) {
  if (!r || !r->data) return "null pointer";
  const int64_t per16 = dtype == DP_BF16 ? 8 : 4, ts = n_tokens > 1 ? r->token_stride : 0, hs = heads > 1 ? r->head_stride : 0;
  if (((uintptr_t)r->data & 15) || ts % per16 || hs % per16) return "rows must be 16-byte aligned, in their strides too";
  if (ts < 0 || hs < 0 || ts > ((int64_t)1 << 38) || hs > ((int64_t)1 << 38)) return "strides must be in [0, 2^38]";
  if (written) {
    const bool by_token = ts >= hs;                       // which of the two steps is the larger
    const int64_t lo = by_token ? hs : ts, hi = by_token ? ts : hs, n_lo = by_token ? heads : n_tokens, n_hi = by_token ? n_tokens : heads;
    if ((n_lo > 1 && lo < head_dim) || (n_hi > 1 && hi < (n_lo > 1 ? (n_lo - 1) * lo : 0) + head_dim)) return "rows that are written must not overlap one another";
  }
  return nullptr;
}
inline int refuse(const char* entry, const char* why) {
  thread_local char text[200];
  snprintf(text, sizeof text, "%s: %s", entry, why);
  return dp_set_error(DP_EINVAL, text);
}
#define REFUSE_IF(expr) do { if (const char* why = (expr)) return refuse(entry, why); } while (0)
