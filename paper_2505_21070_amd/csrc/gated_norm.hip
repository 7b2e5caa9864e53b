// What lies between two branches of a layer, in one pass over the rows (dp_gated_norm): the branch's output, normalised or as it is, gated and added to the
// residual stream, and the stream normalised, modulated or with a gain, for the next branch:
//   x' = x + r * gate * t,  t = y or N(y) * post_gain;   h = N(x') * gain * (1 + scale) + shift
// N is an RMSNorm or a LayerNorm (biased variance, two passes over registers).  Statistics and sums are fp32, h comes from x' before its rounding, and x' and h are
// rounded once.
//
// Bound by memory: x, y, x' and h once each, 12 bytes a value with an fp32 stream and bf16 rows.  A row stays in the registers of the wavefronts that own it, 8
// consecutive values a lane and trip; gate, scale and shift come out of the caches.  6240 rows of 5120, fp32 stream, LayerNorm, modulated 82 us (384 MB, 4.7 TB/s; a copy 5.1); with
// vectors kept in registers over several rows 2 % less at twice the registers, with non-temporal loads 2 % more.  48 rows of 1536 6 us.
#include <math.h>
#include <stdio.h>

#include "../../include/dualparal.h"
#include "common.h"

int dp_set_error(int code, const char* msg);   // defined next to dp_last_error

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct NormArgs {
  const void *x, *y;
  void *xo, *h;
  int64_t x_s, y_s, xo_s, h_s, n;
  const void *gain, *post;
  const float *gate, *scale, *shift;
  const int32_t* group;
  int32_t dim, n_groups, rms;
  float eps, r, inv_dim;
};

// eight consecutive values, as they are in memory and in fp32
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
  u32x4 w;
  __device__ __forceinline__ void load(const void* p, int64_t at) { w = *(const u32x4*)((const bf16_t*)p + at); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ void store(void* p, int64_t at, const float (&v)[8]) {
    *(u32x4*)((bf16_t*)p + at) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  }
};
template <> struct Eight<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const void* p, int64_t at) { a = *(const f32x4*)((const float*)p + at); b = *(const f32x4*)((const float*)p + at + 4); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
  }
  static __device__ __forceinline__ void store(void* p, int64_t at, const float (&v)[8]) {
    *(f32x4*)((float*)p + at) = f32x4{v[0], v[1], v[2], v[3]};
    *(f32x4*)((float*)p + at + 4) = f32x4{v[4], v[5], v[6], v[7]};
  }
};

// the sum over a row of W wavefronts, the same in all of its lanes, added up in wavefront order
template <int W> __device__ __forceinline__ float over_row(float v, float* smem) {
  v = wave_sum(v);
  if constexpr (W > 1) {
    __syncthreads();                       // the sum before this one has been read
    if ((threadIdx.x & 63) == 0) smem[threadIdx.x >> 6] = v;
    __syncthreads();
    v = smem[0];
#pragma unroll
    for (int w = 1; w < W; ++w) v += smem[w];
  }
  return v;
}
// N(v) in place.  Values beyond the row's end do not count and are 0 on entry.
template <int W, int C> __device__ __forceinline__ void normalise(float (&v)[C][8], const bool (&in)[C], const NormArgs& a, float* smem) {
  float sum = 0.f, mean = 0.f;
  if (!a.rms) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += v[c][i];
    mean = over_row<W>(sum, smem) * a.inv_dim;
    sum = 0.f;
  }
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[c][i] = in[c] ? v[c][i] - mean : 0.f;
      sum = fmaf(v[c][i], v[c][i], sum);
    }
  const float inv = rsqrtf(over_row<W>(sum, smem) * a.inv_dim + a.eps);
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[c][i] *= inv;
}

// One row: W wavefronts, C trips of 8 values a lane.  W = 1: four rows a block.
template <typename S, typename T, int W, int C>
__global__ __launch_bounds__(W == 8 ? 512 : 256) void k_gated_norm(const NormArgs a) {
  __shared__ float smem[W];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row = W == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
  if (row >= a.n) return;
  const int group = a.group ? a.group[row] : 0;
  if ((uint32_t)group >= (uint32_t)a.n_groups) return;        // a row of padding
  int at[C];
  bool in[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int first = ((c * W + (W == 1 ? 0 : wave)) * 64 + lane) * 8;
    in[c] = first < a.dim;
    at[c] = in[c] ? first : 0;                                // beyond the end: read at the beginning, and not used
  }
  const int64_t vec = (int64_t)group * a.dim;
  Eight<S> xr[C];
  Eight<T> yr[C];
#pragma unroll
  for (int c = 0; c < C; ++c) xr[c].load(a.x, row * a.x_s + at[c]);
  if (a.y) {
#pragma unroll
    for (int c = 0; c < C; ++c) yr[c].load(a.y, row * a.y_s + at[c]);
  }
  float x[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    xr[c].get(x[c]);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[c][i] = in[c] ? x[c][i] : 0.f;
  }
  if (a.y) {
    float t[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      yr[c].get(t[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) t[c][i] = in[c] ? t[c][i] : 0.f;
    }
    if (a.post) {
      normalise<W, C>(t, in, a, smem);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        Eight<T> g;
        float v[8];
        g.load(a.post, at[c]);
        g.get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) t[c][i] *= v[i];
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (a.gate) {
        Eight<float> g;
        float v[8];
        g.load(a.gate, vec + at[c]);
        g.get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[c][i] = in[c] ? fmaf(a.r * v[i], t[c][i], x[c][i]) : 0.f;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[c][i] = fmaf(a.r, t[c][i], x[c][i]);
      }
      if (a.xo && in[c]) Eight<S>::store(a.xo, row * a.xo_s + at[c], x[c]);
    }
  }
  if (!a.h) return;
  normalise<W, C>(x, in, a, smem);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (a.gain) {
      Eight<T> g;
      float v[8];
      g.load(a.gain, at[c]);
      g.get(v);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[c][i] *= v[i];
    }
    if (a.scale) {
      Eight<float> m, s;
      float mv[8], sv[8];
      m.load(a.scale, vec + at[c]);
      s.load(a.shift, vec + at[c]);
      m.get(mv);
      s.get(sv);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[c][i] = fmaf(x[c][i], 1.f + mv[i], sv[i]);
    }
    if (in[c]) Eight<T>::store(a.h, row * a.h_s + at[c], x[c]);
  }
}

template <typename S, typename T> void launch(const NormArgs& a, hipStream_t st) {
  const unsigned g1 = (unsigned)((a.n + 3) / 4), g = (unsigned)a.n;
  const int chunks = (a.dim + 511) / 512;                      // of 512 values
#define ONE(C) k_gated_norm<S, T, 1, C><<<g1, 256, 0, st>>>(a)
#define FOUR(C) k_gated_norm<S, T, 4, C><<<g, 256, 0, st>>>(a)
#define EIGHT(C) k_gated_norm<S, T, 8, C><<<g, 512, 0, st>>>(a)
  if (chunks == 1) ONE(1); else if (chunks == 2) ONE(2); else if (chunks == 3) ONE(3); else if (chunks == 4) ONE(4);
  else if (chunks <= 8) FOUR(2); else if (chunks <= 12) FOUR(3); else if (chunks <= 16) FOUR(4);
  else if (chunks <= 24) EIGHT(3); else EIGHT(4);
#undef ONE
#undef FOUR
#undef EIGHT
}

int refuse_norm(const char* why) {
  thread_local char text[200];
  snprintf(text, sizeof text, "dp_gated_norm: %s", why);
  return dp_set_error(DP_EINVAL, text);
}
const char* why_not_2d(const void* p, int64_t stride, int64_t n, int32_t dim, int32_t dtype, bool written) {
  const int64_t per16 = dtype == DP_BF16 ? 8 : 4, s = n > 1 ? stride : 0;
  if (((uintptr_t)p & 15) || s % per16) return "rows must be 16-byte aligned, in their stride too";
  if (s < 0 || s > ((int64_t)1 << 38)) return "strides must be in [0, 2^38]";
  if (written && n > 1 && s < dim) return "rows that are written must not overlap one another";
  return nullptr;
}

}  // namespace

extern "C" int dp_gated_norm(const dp_gated_norm_config* c, const void* x, int64_t x_stride, const void* y, int64_t y_stride, int64_t n, void* x_out,
                             int64_t x_out_stride, void* h, int64_t h_stride, void* stream) {
#define REFUSE_IF(expr) do { if (const char* why = (expr)) return refuse_norm(why); } while (0)
  REFUSE_IF(!c ? "null pointer" : nullptr);
  REFUSE_IF(c->dim < 8 || c->dim > 16384 || c->dim % 8 ? "dim must be a multiple of 8 in [8, 16384]" : nullptr);
  REFUSE_IF(c->dtype != DP_F32 && c->dtype != DP_BF16 ? "dtype must be DP_F32 or DP_BF16" : nullptr);
  REFUSE_IF(c->stream_dtype != DP_F32 && c->stream_dtype != c->dtype ? "stream_dtype must be DP_F32 or dtype" : nullptr);
  REFUSE_IF(c->norm != DP_NORM_LAYER && c->norm != DP_NORM_RMS ? "norm must be DP_NORM_LAYER or DP_NORM_RMS" : nullptr);
  REFUSE_IF(c->n_groups < 1 ? "n_groups must be at least 1" : nullptr);
  REFUSE_IF(!(c->eps >= 0.f && c->eps < INFINITY) ? "eps must be finite and not negative" : nullptr);
  REFUSE_IF(!(fabsf(c->res_scale) < INFINITY) ? "res_scale must be finite" : nullptr);
  REFUSE_IF((c->scale != nullptr) != (c->shift != nullptr) ? "scale and shift go together" : nullptr);
  REFUSE_IF(((uintptr_t)c->gain | (uintptr_t)c->post_gain | (uintptr_t)c->gate | (uintptr_t)c->scale | (uintptr_t)c->shift) & 15 ? "gains, gates, scales and shifts must be 16-byte aligned" : nullptr);
  REFUSE_IF((uintptr_t)c->group & 3 ? "group must be 4-byte aligned" : nullptr);
  // launches stay below 2^32 threads: 256 a row of more than 2048 values, 512 of more than 8192
  REFUSE_IF(n < 0 || n > (1 << 24) || n * c->dim > (int64_t)1 << 35 ? "n must be in [0, 2^24], n * dim at most 2^35" : nullptr);
  if (n == 0) return DP_OK;
  REFUSE_IF(!x || (!y && !h) ? "null pointer" : nullptr);
  REFUSE_IF(!y && (x_out || c->post_gain || c->gate) ? "x_out, post_gain and gate go with y" : nullptr);
  REFUSE_IF(!h && (c->gain || c->scale) ? "gain, scale and shift go with h" : nullptr);
  REFUSE_IF(!h && !x_out ? "nothing to write" : nullptr);
  REFUSE_IF(h == x_out ? "x_out and h must not be the same" : nullptr);
  REFUSE_IF(why_not_2d(x, x_stride, n, c->dim, c->stream_dtype, false));
  if (y) REFUSE_IF(why_not_2d(y, y_stride, n, c->dim, c->dtype, false));
  if (x_out) REFUSE_IF(why_not_2d(x_out, x_out_stride, n, c->dim, c->stream_dtype, true));
  if (h) REFUSE_IF(why_not_2d(h, h_stride, n, c->dim, c->dtype, true));
#undef REFUSE_IF
  NormArgs a{};
  a.x = x; a.y = y; a.xo = x_out; a.h = h;
  a.x_s = x_stride; a.y_s = y_stride; a.xo_s = x_out_stride; a.h_s = h_stride; a.n = n;
  a.gain = c->gain; a.post = c->post_gain; a.gate = c->gate; a.scale = c->scale; a.shift = c->shift; a.group = c->group;
  a.dim = c->dim; a.n_groups = c->n_groups; a.rms = c->norm == DP_NORM_RMS; a.eps = c->eps; a.r = c->res_scale; a.inv_dim = 1.f / (float)c->dim;
  const hipStream_t st = (hipStream_t)stream;
  (void)hipGetLastError();
  if (c->dtype == DP_F32) launch<float, float>(a, st);
  else if (c->stream_dtype == DP_F32) launch<float, bf16_t>(a, st);
  else launch<bf16_t, bf16_t>(a, st);
  if (hipGetLastError() != hipSuccess) return dp_set_error(DP_EHIP, "dp_gated_norm: the launch failed");
  return DP_OK;
}
