// Products with weights held in 4 bits (dp_linear_fp4): y = act(x W^T + b), and the way of a matrix into 4 bits (dp_fp4_pack).
//
// Weights are read as they are held and become bf16 in registers, exactly, two codes an instruction, just before they are the A operand of
// v_mfma_f32_16x16x32_bf16: 16 outputs of a row tile against 16 tokens.  fp32 inputs are split into three bf16 parts of 8 bits each, which together are
// the input exactly (as far as bf16 reaches down: a part below 2^-126 may be lost), so that fp32 takes the same instructions three times instead of ones of 1/16 the rate; all sums are fp32.
//
// The order of the products' k is free, as long as both operands have the same: a lane takes consecutive codes of one row, whole groups, and the values of the
// token that meet them.
#include <math.h>
#include <stdio.h>

#include <atomic>

#include "../../include/dualparal.h"
#include "fp4.h"
#include "kernels.h"

int dp_set_error(int code, const char* msg);   // defined next to dp_last_error

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

struct LinearArgs {
  const uint8_t *codes, *scales;
  const void *bias, *x;
  void* y;
  int64_t x_s, y_s, n;
  int32_t in, out, act;
  int32_t row_tiles, token_tiles;          // k_many: of a block's rows and tokens
  int32_t by_four;                         // outputs may be stored four at a time
};

__device__ __forceinline__ float activated(float v, int act) {
  if (act == DP_ACT_GELU) v = v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-2.f * 0.7978845608028654f * 1.4426950408889634f * fmaf(0.044715f * v * v, v, v)));
  if (act == DP_ACT_SILU) v = v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * v));
  return v;
}

// Eight values of a token as B operands: one for bf16, the three parts of fp32 values, each the upper 16 bits of what is left.  CAREFUL: of a value that is not
// finite there is no rest.
template <typename T> struct Parts;
template <> struct Parts<bf16_t> {
  static constexpr int N = 1;
  typedef uint4 Raw;                       // eight values as they are in memory
  template <bool CAREFUL> static __device__ __forceinline__ void split(const Raw& r, bf16x8 (&p)[1]) { p[0] = __builtin_bit_cast(bf16x8, r); }
};
struct Raw8 { f32x4 a, b; };
template <> struct Parts<float> {
  static constexpr int N = 3;
  typedef Raw8 Raw;
  template <bool CAREFUL> static __device__ __forceinline__ void split(const Raw& r, bf16x8 (&p)[3]) {
    uint32_t w[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[2] = {i < 2 ? r.a[2 * i] : r.b[2 * i - 4], i < 2 ? r.a[2 * i + 1] : r.b[2 * i - 3]};
#pragma unroll
      for (int j = 0; j < 3; ++j) {
        w[j][i] = __builtin_amdgcn_perm(__float_as_uint(v[1]), __float_as_uint(v[0]), 0x07060302u);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float rest = v[h] - __uint_as_float(__float_as_uint(v[h]) & 0xffff0000u);
          v[h] = CAREFUL && !(fabsf(v[h]) < INFINITY) ? 0.f : rest;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 3; ++j) p[j] = __builtin_bit_cast(bf16x8, make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]));
  }
};
__device__ __forceinline__ void zero(uint4& v) { v = uint4{}; }
__device__ __forceinline__ void zero(Raw8& v) { v.a = v.b = f32x4{0.f, 0.f, 0.f, 0.f}; }
__device__ __forceinline__ bool finite(f32x4 v) { return fmaf(v[0], 0.f, v[1] * 0.f) + fmaf(v[2], 0.f, v[3] * 0.f) == 0.f; }

// Few tokens: R * 16 outputs, NT * 16 tokens, W wavefronts that deal the inputs out in steps of 256 (wavefront w: steps w, w + W, ..) and add up in LDS in
// wavefront order.  A lane takes 64 consecutive codes of a row, two groups, a step.  Bound by the codes' way from memory: two steps are on their way.
template <typename T, int R, int NT, int W>
__global__ __launch_bounds__(W * 64) void k_few(const LinearArgs a) {
  typedef Parts<T> P;
  __shared__ f32x4 sums[W][R * NT][64];
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row0 = blockIdx.x * (R * 16), groups = a.in / FP4_GROUP, steps = (a.in + 255) / 256;
  const uint8_t* codes[R];
  const uint8_t* scales[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = row0 + r * 16 + lr < a.out ? row0 + r * 16 + lr : a.out - 1;
    codes[r] = a.codes + (int64_t)row * (a.in / 2) + lg * 32;
    scales[r] = a.scales + (int64_t)row * groups + lg * 2;
  }
  const T* x[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int64_t token = t * 16 + lr < a.n ? t * 16 + lr : a.n - 1;
    x[t] = (const T*)a.x + token * a.x_s + lg * 64;
  }
  struct Step { uint4 c[R][2]; uint32_t s[R][2]; };
  auto load = [&](Step& s, int step) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool in = step * 8 + lg * 2 + h < groups;
        s.c[r][h] = in ? *(const uint4*)(codes[r] + (int64_t)step * 128 + h * 16) : uint4{};
        s.s[r][h] = in ? scales[r][step * 8 + h] : 127u;
      }
  };
  f32x4 acc[R][NT];
  auto multiply = [&](const Step& s, int step, auto careful) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool in = step * 8 + lg * 2 + h < groups;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bf16x8 w[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const uint32_t c = i == 0 ? s.c[r][h].x : i == 1 ? s.c[r][h].y : i == 2 ? s.c[r][h].z : s.c[r][h].w;
          w[r] = __builtin_bit_cast(bf16x8, fp4x8_to_bf16(c, __uint_as_float(s.s[r][h] << 23)));
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          typename P::Raw raw;
          if (in) raw = *(const typename P::Raw*)(x[t] + step * 256 + h * 32 + i * 8); else zero(raw);
          bf16x8 p[P::N];
          P::template split<decltype(careful)::value>(raw, p);
#pragma unroll
          for (int j = 0; j < P::N; ++j)
#pragma unroll
            for (int r = 0; r < R; ++r) acc[r][t] = mfma(w[r], p[j], acc[r][t]);
        }
      }
    }
  };
  auto all = [&](auto careful) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    Step s0, s1;
    int step = wave;
    if (step < steps) load(s0, step);
    if (step + W < steps) load(s1, step + W);
    while (step < steps) {
      const Step now = s0;
      s0 = s1;
      if (step + 2 * W < steps) load(s1, step + 2 * W);
      multiply(now, step, careful);
      step += W;
    }
  };
  all(std::false_type{});
  if constexpr (P::N > 1) {                // what is not finite has parts that are not: once more with a look at each value
    bool fine = true;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t) fine &= finite(acc[r][t]);
    if (!__all(fine)) all(std::true_type{});
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t) sums[wave][r * NT + t][lane] = acc[r][t];
  __syncthreads();
  for (int i = threadIdx.x; i < R * NT * 256; i += W * 64) {
    const int token = i / (R * 16), of = i % (R * 16), tile = of / 16 * NT + token / 16, at = (of % 16 / 4) * 16 + token % 16;
    if (token >= a.n || row0 + of >= a.out) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += sums[w][tile][at][of & 3];
    if (a.bias) v += Elem<T>::ld((const T*)a.bias + row0 + of);
    Elem<T>::st((T*)a.y + token * a.y_s + row0 + of, activated(v, a.act));
  }
}

// Many tokens: four wavefronts of R * 16 outputs each, side by side, that share NT * 16 tokens' inputs in LDS, in steps of 128; codes go straight into
// registers.  LDS rows of a token are 128 inputs, their 16-byte chunks exchanged by the row so that 16 rows of one chunk column spread over the banks.  Inputs
// come by direct loads, two stages.
template <typename T, int R, int NT>
__global__ __launch_bounds__(256) void k_many(const LinearArgs a) {
  typedef Parts<T> P;
  constexpr int ROW = 128 * sizeof(T), CPR = ROW / 16, TOKENS = NT * 16, TILE = TOKENS * ROW, TRIPS = TILE / (256 * 16);
  __shared__ __align__(16) char smem[2][TILE];
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // blocks are handed out to the eight XCDs in turn: each gets a run of tiles, whose neighbours share weights
  const int total = a.row_tiles * a.token_tiles, per = (total + 7) >> 3, pid = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || pid >= total) return;
  const int row0 = pid / a.token_tiles * (R * 64) + wave * (R * 16), groups = a.in / FP4_GROUP, steps = (a.in + 127) / 128;
  const int64_t token0 = (int64_t)(pid % a.token_tiles) * TOKENS;
  const int tokens = a.n - token0 < TOKENS ? (int)(a.n - token0) : TOKENS;
  const uint8_t* codes[R];
  const uint8_t* scales[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = row0 + r * 16 + lr < a.out ? row0 + r * 16 + lr : a.out - 1;
    codes[r] = a.codes + (int64_t)row * (a.in / 2) + lg * 16;
    scales[r] = a.scales + (int64_t)row * groups + lg;
  }
  // this lane's chunk of a trip: LDS place (trip * 256 + thread) holds row place / CPR, chunk place % CPR exchanged by the row
  const T* const x = (const T*)a.x + token0 * a.x_s;
  const uint32_t x_bytes = (uint32_t)(((int64_t)(tokens - 1) * a.x_s + a.in) * sizeof(T));
  uint32_t from[TRIPS];
  int chunk[TRIPS];
#pragma unroll
  for (int i = 0; i < TRIPS; ++i) {
    const int place = i * 256 + (int)threadIdx.x, row = place / CPR;
    chunk[i] = place % CPR ^ (row & 15);
    from[i] = (uint32_t)((row < tokens ? row : 0) * a.x_s * sizeof(T)) + chunk[i] * 16;   // rows of no token: the first one's, not stored
  }
  auto move = [&](int step, int stage) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TRIPS; ++i) {
      // the last step's inputs beyond the row's end are zeros, not the next row's
      const uint32_t at = step * ROW + chunk[i] * 16 < a.in * (int)sizeof(T) ? from[i] + step * ROW : 0x80000000u;
      load_lds16(x, x_bytes, at, 0, (uint4*)(smem[stage] + (i * 4 + wave) * 1024));
    }
  };
  struct Step { uint4 c[R]; uint32_t s[R]; };
  auto load = [&](Step& s, int step) __attribute__((always_inline)) {
    const bool in = step * 4 + lg < groups;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s.c[r] = in ? *(const uint4*)(codes[r] + (int64_t)step * 64) : uint4{};
      s.s[r] = in ? scales[r][step * 4] : 127u;
    }
  };
  f32x4 acc[R][NT];
  auto multiply = [&](const Step& s, const char* tile, auto careful) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x8 w[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const uint32_t c = i == 0 ? s.c[r].x : i == 1 ? s.c[r].y : i == 2 ? s.c[r].z : s.c[r].w;
        w[r] = __builtin_bit_cast(bf16x8, fp4x8_to_bf16(c, __uint_as_float(s.s[r] << 23)));
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const char* const row = tile + (t * 16 + lr) * ROW;
        typename P::Raw raw;
        if constexpr (P::N == 1) raw = *(const uint4*)(row + ((lg * 4 + i) ^ lr) * 16);
        else { raw.a = *(const f32x4*)(row + ((lg * 8 + i * 2) ^ lr) * 16); raw.b = *(const f32x4*)(row + ((lg * 8 + i * 2 + 1) ^ lr) * 16); }
        bf16x8 p[P::N];
        P::template split<decltype(careful)::value>(raw, p);
#pragma unroll
        for (int j = 0; j < P::N; ++j)
#pragma unroll
          for (int r = 0; r < R; ++r) acc[r][t] = mfma(w[r], p[j], acc[r][t]);
      }
    }
  };
  auto all = [&](auto careful) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    Step next;
    move(0, 0);
    load(next, 0);
    for (int step = 0; step < steps; ++step) {
      tile_barrier();                      // this step's inputs are there, and all are done with the other stage
      const Step now = next;
      if (step + 1 < steps) {
        move(step + 1, (step + 1) & 1);
        load(next, step + 1);
      }
      multiply(now, smem[step & 1], careful);
    }
  };
  all(std::false_type{});
  if constexpr (P::N > 1) {                // what is not finite has parts that are not: once more with a look at each value
    bool fine = true;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t) fine &= finite(acc[r][t]);
    if (__syncthreads_or(!fine)) all(std::true_type{});
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int64_t token = token0 + t * 16 + lr;
    if (token >= a.n) continue;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = row0 + r * 16 + lg * 4;
      T* const to = (T*)a.y + token * a.y_s + row;
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = acc[r][t][i];
        if (a.bias && row + i < a.out) v[i] += Elem<T>::ld((const T*)a.bias + row + i);
        v[i] = activated(v[i], a.act);
      }
      if (a.by_four && row + 3 < a.out) {
        if constexpr (sizeof(T) == 2) *(uint2*)to = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        else *(f32x4*)to = f32x4{v[0], v[1], v[2], v[3]};
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (row + i < a.out) Elem<T>::st(to + i, v[i]);
      }
    }
  }
}

template <typename T, int R, int NT> void few(const LinearArgs& a, hipStream_t st) {
  k_few<T, R, NT, 8><<<(unsigned)((a.out + R * 16 - 1) / (R * 16)), 512, 0, st>>>(a);
}
template <typename T, int R, int NT> void many(LinearArgs& a, hipStream_t st) {
  a.row_tiles = (a.out + R * 64 - 1) / (R * 64);
  a.token_tiles = (int32_t)((a.n + NT * 16 - 1) / (NT * 16));
  const int64_t total = (int64_t)a.row_tiles * a.token_tiles;
  k_many<T, R, NT><<<(unsigned)((total + 7) / 8 * 8), 256, 0, st>>>(a);
}
template <typename T> void launch(LinearArgs& a, hipStream_t st) {
  if (a.n <= 16) few<T, 1, 1>(a, st);
  else if (a.n <= 32) few<T, 1, 2>(a, st);
  else if (a.n <= 64) few<T, 1, 4>(a, st);
  else if constexpr (sizeof(T) == 2) many<T, 4, 8>(a, st);
  else many<T, 4, 4>(a, st);
}

// A group a thread: its 32 values, largest one, byte and codes.
template <typename T> __global__ __launch_bounds__(256) void k_pack(const T* src, int64_t stride, int64_t rows, int32_t groups, uint8_t* codes, uint8_t* scales) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= rows * groups) return;
  const int64_t row = id / groups;
  const T* const from = src + row * stride + (id - row * groups) * FP4_GROUP;
  float v[FP4_GROUP], top = 0.f;
#pragma unroll
  for (int i = 0; i < FP4_GROUP; ++i) {
    v[i] = Elem<T>::ld(from + i);
    top = fmaxf(top, fp4_size(v[i]));
  }
  const uint32_t byte = fp4_byte(top);
  const float inv = fp4_inverse(byte);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = to_fp4x4(v[8 * i], v[8 * i + 1], v[8 * i + 2], v[8 * i + 3], inv) | to_fp4x4(v[8 * i + 4], v[8 * i + 5], v[8 * i + 6], v[8 * i + 7], inv) << 16;
  *(uint4*)(codes + id * (FP4_GROUP / 2)) = make_uint4(w[0], w[1], w[2], w[3]);
  scales[id] = (uint8_t)byte;
}

int refuse_linear(const char* entry, const char* why) {
  thread_local char text[200];
  snprintf(text, sizeof text, "%s: %s", entry, why);
  return dp_set_error(DP_EINVAL, text);
}
const char* why_not_matrix(int32_t out, int32_t in, int32_t dtype, const void* codes, const uint8_t* scales) {
  if (in < FP4_GROUP || in > 1 << 20 || in % FP4_GROUP) return "in must be a multiple of 32 in [32, 2^20]";
  if (out < 1 || out > 1 << 24) return "out must be in [1, 2^24]";
  if (dtype != DP_F32 && dtype != DP_BF16) return "dtype must be DP_F32 or DP_BF16";
  if (!codes || !scales) return "null pointer";
  if ((uintptr_t)codes & 15) return "codes must be 16-byte aligned";
  return nullptr;
}

}  // namespace

extern "C" int dp_fp4_pack(const void* src, int64_t stride, int32_t out, int32_t in, int32_t dtype, void* codes, uint8_t* scales, void* stream) {
  static const char entry[] = "dp_fp4_pack";
  if (const char* why = why_not_matrix(out, in, dtype, codes, scales)) return refuse_linear(entry, why);
  const int size = dtype == DP_BF16 ? 2 : 4;
  if (!src) return refuse_linear(entry, "null pointer");
  if ((uintptr_t)src & (size - 1)) return refuse_linear(entry, "rows must be aligned to their type");
  if (out > 1 && (stride < 0 || stride > (int64_t)1 << 38)) return refuse_linear(entry, "strides must be in [0, 2^38]");
  const int64_t threads = (int64_t)out * (in / FP4_GROUP);
  if (threads > (int64_t)1 << 31) return refuse_linear(entry, "out * in must be at most 2^36");
  const hipStream_t st = (hipStream_t)stream;
  const unsigned g = (unsigned)((threads + 255) / 256);
  (void)hipGetLastError();
  if (dtype == DP_BF16) k_pack<bf16_t><<<g, 256, 0, st>>>((const bf16_t*)src, stride, out, in / FP4_GROUP, (uint8_t*)codes, scales);
  else k_pack<float><<<g, 256, 0, st>>>((const float*)src, stride, out, in / FP4_GROUP, (uint8_t*)codes, scales);
  if (hipGetLastError() != hipSuccess) return dp_set_error(DP_EHIP, "dp_fp4_pack: the launch failed");
  return DP_OK;
}

extern "C" int dp_linear_fp4(const dp_fp4_matrix* w, const void* x, int64_t x_stride, int64_t n, int32_t act, void* y, int64_t y_stride, void* stream) {
  static const char entry[] = "dp_linear_fp4";
#define REFUSE_IF(expr) do { if (const char* why = (expr)) return refuse_linear(entry, why); } while (0)
  REFUSE_IF(!w ? "null pointer" : nullptr);
  REFUSE_IF(why_not_matrix(w->out, w->in, w->dtype, w->codes, w->scales));
  REFUSE_IF(act != DP_ACT_NONE && act != DP_ACT_GELU && act != DP_ACT_SILU ? "act must be DP_ACT_NONE, DP_ACT_GELU or DP_ACT_SILU" : nullptr);
  REFUSE_IF(n < 0 || n > 1 << 24 || n * w->out > (int64_t)1 << 35 ? "n must be in [0, 2^24], n * out at most 2^35" : nullptr);
  if (n == 0) return DP_OK;
  const int size = w->dtype == DP_BF16 ? 2 : 4;
  REFUSE_IF(!x || !y ? "null pointer" : nullptr);
  REFUSE_IF(((uintptr_t)x & 15) || (n > 1 && x_stride % (16 / size)) ? "rows of x must be 16-byte aligned, in their stride too" : nullptr);
  REFUSE_IF(n > 1 && (x_stride < 0 || x_stride > 1 << 22) ? "x_stride must be in [0, 2^22]" : nullptr);
  REFUSE_IF(((uintptr_t)y | (uintptr_t)w->bias) & (size - 1) ? "y and the bias must be aligned to their type" : nullptr);
  REFUSE_IF(n > 1 && (y_stride < w->out || y_stride > (int64_t)1 << 38) ? "y_stride must be in [out, 2^38]" : nullptr);
#undef REFUSE_IF
  LinearArgs a{};
  a.codes = (const uint8_t*)w->codes; a.scales = w->scales; a.bias = w->bias; a.x = x; a.y = y;
  a.x_s = n > 1 ? x_stride : 0; a.y_s = n > 1 ? y_stride : 0; a.n = n; a.in = w->in; a.out = w->out; a.act = act;
  a.by_four = (uintptr_t)y % (4 * size) == 0 && a.y_s % 4 == 0;
  const hipStream_t st = (hipStream_t)stream;
  (void)hipGetLastError();
  if (w->dtype == DP_BF16) launch<bf16_t>(a, st); else launch<float>(a, st);
  if (hipGetLastError() != hipSuccess) return dp_set_error(DP_EHIP, "dp_linear_fp4: the launch failed");
  return DP_OK;
}
