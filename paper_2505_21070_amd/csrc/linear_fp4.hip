// Products with weights held in 4 bits (dp_linear_fp4): y = act(x W^T + b), and the way of a matrix into 4 bits (dp_fp4_pack).
//
// Weights are read as they are held and become bf16 in registers, exactly, two codes an instruction, just before they are the A operand of
// v_mfma_f32_16x16x32_bf16: 16 outputs of a row tile against 16 tokens.  fp32 inputs are split into three bf16 parts of 8 bits each, which together are
// the input exactly (as far as bf16 reaches down: a part below 2^-126 may be lost), so that fp32 takes the same instructions three times instead of ones of 1/16 the rate; all sums are fp32.
//
// What bounds it: a few tokens, the codes' way and the steps' latency around it: one token, 5120 -> 13824, 10.7 us with matrices out of memory, 9.2 with one out of the last-level cache,
// where a kernel that reads as many bytes and no more takes 7.0 and 4.2 (16 tokens 11.6 and 9.2).  Some 20 to 500 tokens, conversions and reads of LDS, which each tile of tokens repeats: 48 tokens, 13824 -> 5120, 16 us out of the
// cache (memory 7, products 5), 256 tokens, 5120 -> 5120, 20 (products 10).  Many, the matrix pipes: 6240 tokens, 5120 -> 5120, 256 us, 1.28 PFLOP/s.  fp32 pays three instructions and the splitting, which
// each wavefront repeats: one token, 13824 -> 5120, 29 us (bf16 11 to 13), 48 tokens 47, 1560 tokens, 1536 -> 8960, 127, 338 TFLOP/s.
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
  const uint8_t* laid;
  const void *bias, *x;
  void* y;
  int64_t x_s, y_s, n;
  int32_t in, out, act;
  int32_t row_tiles, token_tiles;          // of a block's rows and tokens
  int32_t parts;                           // ranges of the inputs, whose sums go into partial [parts][n][out]
  float* partial;
  int32_t by_four, by_eight;               // outputs may be stored four at a time, eight (rows end with a whole eight)
};

__device__ __forceinline__ float activated(float v, int act) {
  constexpr float C = -2.f * 0.7978845608028654f * 1.4426950408889634f;
  if (act == DP_ACT_GELU) v = v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * fmaf(C * 0.044715f, v * v, C)));
  if (act == DP_ACT_SILU) v = v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * v));
  return v;
}

// Eight values of a token as B operands: one for bf16, the three parts of fp32 values, each the upper 16 bits of what is left.  CAREFUL: of a value that is not
// finite there is no rest, and NaN is one that its upper 16 bits show.
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
      if (CAREFUL)
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h] = v[h] != v[h] ? __uint_as_float(0x7fc00000u) : v[h];
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
__device__ __forceinline__ bool finite(f32x4 v) { return fmaf(v[0], 0.f, v[1] * 0.f) + fmaf(v[2], 0.f, v[3] * 0.f) == 0.f; }

// Weights as dp_fp4_lay leaves them: for each tile of 16 rows and step of 128 inputs, one behind the other, 1024 bytes of codes and 64 of group bytes.  Codes lie as
// the operands want them: lane l takes 16 bytes, whose word i has the eight codes of row l % 16 that product i (inputs 32 i ..) takes from it (8 (l / 16) ..), and the
// row's four group bytes.  Rows and inputs that fill the last tile and step up are zeros.  Read row by row, the group bytes alone took as long as the codes
// (13824 x 5120, one token: 16 us), since a wavefront's 64 bytes lay in 16 places.
constexpr int CHUNK = 1088;
template <int R> struct Step {
  uint4 c[R];
  uint32_t s[R];
  // laid: the tiles' first chunks (uniform); codes, bytes: the lane's places in a chunk
  __device__ __forceinline__ void load(const uint8_t* const (&laid)[R], int step, uint32_t codes, uint32_t bytes) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint8_t* const at = laid[r] + (int64_t)step * CHUNK;
      c[r] = *(const uint4*)(at + codes);
      s[r] = *(const uint32_t*)(at + bytes);
    }
  }
};
// eight weights: word i with the i-th byte of the row's four
__device__ __forceinline__ bf16x8 weights(uint4 c, uint32_t bytes, int i) {
  const uint32_t w = i == 0 ? c.x : i == 1 ? c.y : i == 2 ? c.z : c.w;
  return __builtin_bit_cast(bf16x8, fp4x8_to_bf16(w, __uint_as_float((bytes >> (8 * i) & 255u) << 23)));
}

// LDS by typed address.  Tiles arrive by direct loads while others are read; what says that the two do not meet are the restricted pointers of `round`, without
// which the compiler has every read of LDS wait for all loads on their way.
typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ u32x4 lds_get(const lds_char* p) {
#ifdef __HIP_DEVICE_COMPILE__
  return *(const __attribute__((address_space(3))) u32x4*)p;
#else
  return u32x4{};
#endif
}

// WK groups of WR x WT wavefronts.  A group has WR * R * 16 outputs and WT * NT * 16 tokens, R and NT tiles of 16 a wavefront; it goes through the inputs in steps of
// 128 (group k: steps k, k + WK, ..), and the groups add up in LDS in their order.  A group's tokens share their inputs through LDS, where they come by direct
// loads; codes go straight into registers.  Either is NS - 1 steps ahead.  LDS rows are a token's 128 inputs, their 16-byte chunks exchanged by the row so that 16
// rows of one chunk column spread over the banks.
template <typename T, int R, int NT, int WR, int WT, int WK, int NS>
__global__ __launch_bounds__(WR * WT * WK * 64) void k_linear(const LinearArgs a) {
  typedef Parts<T> P;
  constexpr int WG = WR * WT, W = WG * WK, ROW = 128 * sizeof(T), CPR = ROW / 16, TOKENS = WT * NT * 16, TILE = TOKENS * ROW, TRIPS = TILE / (WG * 1024), CA = NS - 1;
  static_assert(TRIPS * WG * 1024 == TILE && (NS - 2) * (TRIPS + 2 * R) < 64, "whole trips, which the counter of loads can tell apart");
  extern __shared__ uint4 lds[];
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wg = wave % WG, kg = wave / WG;
  lds_char* const smem = (lds_char*)(lds_void_t*)lds + kg * (NS * TILE);   // the group's NS stages
  // blocks are handed out to the eight XCDs in turn: each gets a run of tiles, whose neighbours share weights
  const int of_part = a.row_tiles * a.token_tiles, total = of_part * a.parts, per = (total + 7) >> 3, id = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || id >= total) return;
  const int part = id / of_part, pid = id - part * of_part;
  const int row0 = pid / a.token_tiles * (WR * R * 16) + wg / WT * (R * 16), all_steps = (a.in + 127) / 128;
  const int step0 = (int)((int64_t)all_steps * part / a.parts), steps = (int)((int64_t)all_steps * (part + 1) / a.parts);
  const int64_t token0 = (int64_t)(pid % a.token_tiles) * TOKENS;
  const int tokens = a.n - token0 < TOKENS ? (int)(a.n - token0) : TOKENS, mine = wg % WT * (NT * 16);
  // tiles beyond the last row: the last one again, not stored
  const int tiles = (a.out + 15) / 16, tile0 = row0 / 16;
  const uint8_t* laid[R];
#pragma unroll
  for (int r = 0; r < R; ++r) laid[r] = a.laid + (int64_t)(tile0 + r < tiles ? tile0 + r : tiles - 1) * all_steps * CHUNK;
  const uint32_t codes_at = lane * 16, bytes_at = 1024 + lr * 4;
  // this lane's chunk of a trip: LDS place (trip * threads + thread) holds row place / CPR, chunk place % CPR exchanged by the row; rows of no token are zeros
  const T* const x = (const T*)a.x + token0 * a.x_s;
  const uint32_t x_bytes = (uint32_t)(((int64_t)(tokens - 1) * a.x_s + a.in) * sizeof(T));
  uint32_t from[TRIPS];
  int in_row[TRIPS];                       // bytes from the chunk on to the row's end, at step 0
#pragma unroll
  for (int i = 0; i < TRIPS; ++i) {
    const int place = (i * WG + wg) * 64 + lane, row = place / CPR, c = (place % CPR ^ (row & 15)) * 16;
    from[i] = row < tokens ? (uint32_t)(row * a.x_s * sizeof(T)) + c : 0x80000000u;
    in_row[i] = a.in * (int)sizeof(T) - c;
  }
  auto move = [&](int step, lds_char* to) __attribute__((always_inline)) {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
    for (int i = 0; i < TRIPS; ++i) {
      const uint32_t at = step * ROW < in_row[i] ? from[i] + step * ROW : 0x80000000u;   // inputs beyond a row's end are zeros, not the next row's
      __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void*)x, 0, (int)x_bytes, 0x00020000), (lds_void_t*)(to + (i * WG + wg) * 1024), 16, at, 0, 0, 0);
    }
#endif
  };
  f32x4 acc[R][NT];
  // The step whose inputs are at `tile`: four products of 32 inputs, whose tokens' operands are read in pieces of NC tiles (which may be of two products), AHEAD pieces before
  // they are used.  Of 64 tokens and two tiles of rows one piece ahead is enough, and leaves registers for a second block on a CU.
  constexpr int NC = NT % 2 == 0 && (NT > 4 || P::N > 1) ? NT / 2 : NT > 4 ? 4 : NT, PIECES = 4 * NT / NC, AHEAD = NT * P::N <= (R > 1 && P::N == 1 ? 3 : 4) ? 3 : 1;
  static_assert(4 * NT % NC == 0, "whole pieces");
  auto multiply = [&](const Step<R>& s, const lds_char* __restrict__ tile, auto careful) __attribute__((always_inline)) {
    const lds_char* const base = tile + (mine + lr) * ROW;
    typename P::Raw raw[AHEAD + 1][NC];
    auto read = [&](int piece) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < NC; ++t) {
        const int i = (piece * NC + t) / NT;
        const lds_char* const row = base + (piece * NC + t) % NT * 16 * ROW;
        auto& to = raw[piece % (AHEAD + 1)][t];
        if constexpr (P::N == 1) to = __builtin_bit_cast(uint4, lds_get(row + ((i * 4 + lg) ^ lr) * 16));
        else { to.a = __builtin_bit_cast(f32x4, lds_get(row + ((i * 8 + lg * 2) ^ lr) * 16)); to.b = __builtin_bit_cast(f32x4, lds_get(row + ((i * 8 + lg * 2 + 1) ^ lr) * 16)); }
      }
    };
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) read(p);
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 w[R];
#pragma unroll
    for (int piece = 0; piece < PIECES; ++piece) {
      if (piece + AHEAD < PIECES) {
        read(piece + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int t = 0; t < NC; ++t) {
        const int i = (piece * NC + t) / NT, tt = (piece * NC + t) % NT;
        if (tt == 0) {
#pragma unroll
          for (int r = 0; r < R; ++r) w[r] = weights(s.c[r], s.s[r], i);
        }
        bf16x8 p[P::N];
        P::template split<decltype(careful)::value>(raw[piece % (AHEAD + 1)][t], p);
#pragma unroll
        for (int j = 0; j < P::N; ++j)
#pragma unroll
          for (int r = 0; r < R; ++r) acc[r][tt] = mfma(w[r], p[j], acc[r][tt]);
      }
    }
  };
  auto arrived = [&](auto behind) __attribute__((always_inline)) {   // at most so many loads are on their way, and all wavefronts are here
    __builtin_amdgcn_sched_barrier(0);
    vm_wait<decltype(behind)::value>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  // A round issues a step's codes and bytes (2 R loads), then a step's inputs (TRIPS): so many loads are behind the inputs of the next step.  Steps past the end:
  // the first one again, never used.
  typedef std::integral_constant<int, (NS - 2) * (TRIPS + 2 * R)> Behind;
  auto round = [&](Step<R>& slot, int step, const lds_char* __restrict__ tile, lds_char* __restrict__ to, auto careful) __attribute__((always_inline)) {
    const Step<R> now = slot;
    const int next = step + CA * WK < steps ? step + CA * WK : step0;
    slot.load(laid, next, codes_at, bytes_at);
    __builtin_amdgcn_sched_barrier(0);
    move(next, to);
    __builtin_amdgcn_sched_barrier(0);
    if (WK == 1 || step < steps) multiply(now, tile, careful);
    arrived(Behind{});
  };
  auto all = [&](auto careful) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (step0 < steps) {
      Step<R> ring[CA];
#pragma unroll
      for (int d = 0; d < CA; ++d) {
        const int step = step0 + kg + d * WK < steps ? step0 + kg + d * WK : step0;
        ring[d].load(laid, step, codes_at, bytes_at);
        __builtin_amdgcn_sched_barrier(0);
        move(step, smem + d * TILE);
        __builtin_amdgcn_sched_barrier(0);
      }
      arrived(Behind{});
      int stage = 0, to = CA;
      for (int step = step0; step < steps; step += CA * WK)
#pragma unroll
        for (int d = 0; d < CA; ++d) {
          if (step + d * WK >= steps) break;
          round(ring[d], step + d * WK + kg, smem + stage * TILE, smem + to * TILE, careful);
          stage = stage + 1 < NS ? stage + 1 : 0;
          to = to + 1 < NS ? to + 1 : 0;
        }
      arrived(std::integral_constant<int, 0>{});   // nothing lands in LDS any more
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
  if constexpr (WK > 1) {
    // sums of a group's tiles behind those of the others; each group adds up and stores its share of the tiles
    static_assert((int)sizeof(f32x4) * 64 * R * NT * W <= NS * TILE * WK, "sums fit where the stages were");
    f32x4* const sums = (f32x4*)lds;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t) sums[(wave * (R * NT) + r * NT + t) * 64 + lane] = acc[r][t];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t)
        if ((r * NT + t) % WK == kg) {
          f32x4 v = sums[(wg * (R * NT) + r * NT + t) * 64 + lane];
#pragma unroll
          for (int k = 1; k < WK; ++k) v += sums[((k * WG + wg) * (R * NT) + r * NT + t) * 64 + lane];
          acc[r][t] = v;
        }
  }
  if (a.parts > 1) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int64_t token = token0 + mine + t * 16 + lr;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int row = row0 + r * 16 + lg * 4;
        if ((WK > 1 && (r * NT + t) % WK != kg) || token >= a.n || row >= a.out) continue;
        float* const to = a.partial + ((int64_t)part * a.n + token) * a.out + row;
        if (a.out % 4 == 0) *(f32x4*)to = acc[r][t];
        else
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (row + i < a.out) to[i] = acc[r][t][i];
      }
    }
    return;
  }
  f32x4 bias[R];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = row0 + r * 16 + lg * 4 + i;
      bias[r][i] = a.bias && row < a.out ? Elem<T>::ld((const T*)a.bias + row) : 0.f;
    }
  auto finished = [&](int r, int t) __attribute__((always_inline)) {
    f32x4 v = acc[r][t] + bias[r];
    if (a.act != DP_ACT_NONE)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = activated(v[i], a.act);
    return v;
  };
  // 16-bit outputs of large tiles go through LDS (free by now, a wavefront's own part of it), so that global memory sees 32 R bytes of a token at once and not 32.  Units of
  // four outputs are exchanged by the token.
  if constexpr (sizeof(T) == 2 && WK == 1 && R > 1) {
    if (a.by_eight) {
      constexpr int UPR = R * 4, CPT = R * 2, PER = 64 / CPT;      // units and 16-byte chunks of a token, tokens of a trip
      static_assert(UPR <= 16 && W * NT * 16 * UPR * 8 <= NS * TILE, "tiles fit where the stages were");
      uint2* const stg = (uint2*)lds + wave * (NT * 16 * UPR);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        __builtin_amdgcn_sched_barrier(0);   // one tile of tokens after the other: registers are full
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const f32x4 v = finished(r, t);
          stg[(t * 16 + lr) * UPR + ((r * 4 + lg) ^ (lr & (UPR - 1)))] = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        }
      }
#pragma unroll
      for (int i = 0; i < NT * 16 / PER; ++i) {
        const int t = i * PER + lane / CPT, ch = lane % CPT;
        uint4 v = ((const uint4*)stg)[t * CPT + ch];
        if (t & 1) v = make_uint4(v.z, v.w, v.x, v.y);
        const int row = row0 + (ch ^ ((t & (UPR - 1)) >> 1)) * 8;
        if (token0 + mine + t < a.n && row < a.out) *(uint4*)((T*)a.y + (token0 + mine + t) * a.y_s + row) = v;
      }
      return;
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int64_t token = token0 + mine + t * 16 + lr;
    if (token >= a.n) continue;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (WK > 1 && (r * NT + t) % WK != kg) continue;
      const int row = row0 + r * 16 + lg * 4;
      T* const to = (T*)a.y + token * a.y_s + row;
      const f32x4 v = finished(r, t);
      if (a.by_four && row + 3 < a.out) {
        if constexpr (sizeof(T) == 2) *(uint2*)to = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        else *(f32x4*)to = v;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (row + i < a.out) Elem<T>::st(to + i, v[i]);
      }
    }
  }
}
// the ranges' sums, in their order
template <typename T> __global__ __launch_bounds__(256) void k_join(const LinearArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, all = a.n * a.out;
  if (i >= all) return;
  float v = 0.f;
#pragma unroll 4
  for (int p = 0; p < a.parts; ++p) v += a.partial[p * all + i];
  const int64_t token = i / a.out, of = i - token * a.out;
  if (a.bias) v += Elem<T>::ld((const T*)a.bias + of);
  Elem<T>::st((T*)a.y + token * a.y_s + of, activated(v, a.act));
}

template <typename T, int R, int NT, int WR, int WT, int WK, int NS> void launch_tiles(LinearArgs& a, hipStream_t st) {
  constexpr int lds = NS * WK * WT * NT * 16 * 128 * (int)sizeof(T);
  static std::atomic<uint64_t> done;
  allow_dynamic_lds((const void*)k_linear<T, R, NT, WR, WT, WK, NS>, lds, done);
  a.row_tiles = (a.out + WR * R * 16 - 1) / (WR * R * 16);
  a.token_tiles = (int32_t)((a.n + WT * NT * 16 - 1) / (WT * NT * 16));
  const int64_t total = (int64_t)a.row_tiles * a.token_tiles * a.parts;
  k_linear<T, R, NT, WR, WT, WK, NS><<<(unsigned)((total + 7) / 8 * 8), WR * WT * WK * 64, lds, st>>>(a);
  if (a.parts > 1) k_join<T><<<(unsigned)((a.n * a.out + 255) / 256), 256, 0, st>>>(a);
}
// The tiles there are, and what they take: rows and tokens of a block, its groups (WK), how many of them a CU holds, and in units of 10 ns a group's step with 1, 2 .. blocks
// on a CU in the last round of blocks, in the rounds before it, and what is done around the steps.  Fitted to some 2600 launches: 512 .. 13824 outputs, 1504 .. 13824 inputs, 1 .. 6240
// tokens.  Against the best tile measured, what the estimate below takes with these constants is 1.0 % slower on average over 95 shapes in bf16 and 0.6 % over 79 in fp32; at worst 23 % (1200 tokens, 5120 ->
// 5120: tiles of 128 x 64 83 us, of 128 x 48 68), 18 % (48 tokens, 1536 -> 8960), 10 %.  A remainder of blocks behind a full round is charged as one block a CU, while places come free in pairs.
// Tiles of tokens in steps of 16 or 32 are worth their code where a round of blocks ends
// just so: 1560 tokens, 8960 -> 1536, 46 us, with 64, 128, 192 and 256 alone 99; 800 tokens, 5120 -> 5120, 45 and 68; 1560 tokens, 1536 -> 8960, 39 and 42; fp32, 1560 tokens, 1536 -> 1536, 33 and 41.
struct Tile { int rows, tokens, groups, per_cu, last[3], full, around; };
#define TILES_BF16(X) \
  X(1, 1, 2, 1, 4, 3, {32, 16, 4, 3, {32, 64, 95}, 88, 152}) \
  X(1, 1, 2, 1, 8, 3, {32, 16, 8, 1, {53}, 70, 214}) \
  X(1, 1, 4, 1, 4, 4, {64, 16, 4, 2, {44, 103}, 103, 219}) \
  X(1, 2, 2, 1, 4, 3, {32, 32, 4, 1, {46}, 51, 175}) \
  X(1, 2, 4, 1, 4, 3, {64, 32, 4, 1, {57}, 62, 251}) \
  X(1, 3, 2, 1, 4, 3, {32, 48, 4, 1, {68}, 82, 207}) \
  X(1, 3, 4, 1, 4, 3, {64, 48, 4, 1, {78}, 94, 301}) \
  X(1, 4, 4, 1, 2, 4, {64, 64, 2, 1, {61}, 67, 213}) \
  X(2, 3, 4, 1, 2, 2, {128, 48, 2, 2, {82, 144}, 150, 181}) \
  X(2, 4, 4, 1, 2, 2, {128, 64, 2, 2, {95, 183}, 195, 219}) \
  X(2, 5, 4, 1, 2, 2, {128, 80, 2, 2, {110, 208}, 221, 260}) \
  X(2, 4, 4, 1, 1, 2, {128, 64, 1, 3, {63, 106, 153}, 164, 275}) \
  X(2, 5, 4, 1, 1, 2, {128, 80, 1, 3, {70, 123, 189}, 193, 321}) \
  X(4, 4, 4, 2, 1, 2, {256, 128, 1, 1, {156}, 188, 632}) \
  X(4, 5, 4, 2, 1, 2, {256, 160, 1, 1, {179}, 203, 645}) \
  X(4, 6, 4, 2, 1, 2, {256, 192, 1, 1, {200}, 231, 676}) \
  X(4, 7, 4, 2, 1, 2, {256, 224, 1, 1, {222}, 261, 803}) \
  X(4, 8, 4, 2, 1, 2, {256, 256, 1, 1, {251}, 304, 781})
#define TILES_F32(X) \
  X(1, 1, 1, 1, 8, 2, {16, 16, 8, 1, {117}, 130, 203}) \
  X(1, 1, 2, 1, 4, 3, {32, 16, 4, 1, {108}, 116, 185}) \
  X(1, 1, 4, 1, 4, 2, {64, 16, 4, 1, {177}, 174, 221}) \
  X(1, 2, 4, 1, 2, 3, {64, 32, 2, 1, {162}, 169, 232}) \
  X(2, 2, 4, 1, 2, 2, {128, 32, 2, 2, {209, 395}, 368, 237}) \
  X(2, 3, 4, 1, 2, 2, {128, 48, 2, 1, {281}, 318, 348}) \
  X(2, 2, 4, 1, 1, 3, {128, 32, 1, 3, {122, 206, 301}, 289, 272}) \
  X(2, 3, 4, 1, 1, 2, {128, 48, 1, 3, {167, 279, 419}, 378, 328}) \
  X(4, 2, 4, 1, 1, 2, {256, 32, 1, 2, {163, 297}, 282, 568}) \
  X(4, 3, 4, 1, 1, 2, {256, 48, 1, 2, {213, 387}, 368, 595}) \
  X(8, 2, 2, 1, 1, 2, {256, 32, 1, 2, {251, 278}, 268, 814}) \
  X(6, 2, 4, 2, 1, 2, {384, 64, 1, 1, {352}, 356, 680}) \
  X(8, 2, 4, 2, 1, 2, {512, 64, 1, 1, {437}, 461, 1090})
template <typename T> struct Tiles;
#define X(R, NT, WR, WT, WK, NS, ...) __VA_ARGS__,
template <> struct Tiles<bf16_t> { static constexpr Tile all[] = {TILES_BF16(X)}; };
template <> struct Tiles<float> { static constexpr Tile all[] = {TILES_F32(X)}; };
#undef X
constexpr Tile Tiles<bf16_t>::all[];
constexpr Tile Tiles<float>::all[];

struct Route { int kind, parts; };
// The kind of tile and the ranges by an estimate of the time: rounds of equal blocks.  Ranges, of the smaller tiles alone, cost a launch and their sums, written and read at
// 4.2 TB/s.
template <typename T> Route route(const LinearArgs& a) {
  Route r{};
  int64_t best = INT64_MAX;
  const int64_t steps = (a.in + 127) / 128;
  for (const Tile& k : Tiles<T>::all) {
    const int64_t tiles = ((int64_t)a.out + k.rows - 1) / k.rows * ((a.n + k.tokens - 1) / k.tokens), slots = 256 * k.per_cu;
    for (int parts = 1; parts <= 8; parts *= 2) {
      if (parts > 1 && (k.rows > 128 || steps < parts * k.groups || tiles * parts > slots)) break;
      const int64_t of_group = ((steps + parts - 1) / parts + k.groups - 1) / k.groups, rounds = tiles * parts / slots, rest = tiles * parts % slots;
      int64_t cost = rounds * (of_group * k.full + k.around);
      if (rest > 0) cost += of_group * k.last[(rest - 1) / 256] + k.around;
      if (parts > 1) cost += 260 + parts * a.n * a.out / 5250;
      if (cost < best) { best = cost; r.kind = (int)(&k - Tiles<T>::all); r.parts = parts; }
    }
  }
  return r;
}
size_t partial_bytes(const LinearArgs& a, const Route& r) { return r.parts > 1 ? (size_t)r.parts * a.n * a.out * sizeof(float) : 0; }
template <typename T> void launch(LinearArgs& a, const Route& r, hipStream_t st) {
  a.parts = r.parts;
  int kind = 0;
#define X(R, NT, WR, WT, WK, NS, ...) if (r.kind == kind++) return launch_tiles<T, R, NT, WR, WT, WK, NS>(a, st);
  if constexpr (sizeof(T) == 2) { TILES_BF16(X) } else { TILES_F32(X) }
#undef X
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

// Whether one of eight codes times 2^(byte - 127) is 2^128 or more: 4 and 6 times 2^126, 2 and more times 2^127
__device__ __forceinline__ bool beyond(uint32_t w, uint32_t byte) { return byte == 253 ? (w & w << 1 & 0x44444444u) != 0 : byte == 254 && (w & 0x44444444u); }
// A chunk of a tile and step a wavefront: each lane its 16 bytes, the first 16 lanes the rows' group bytes.  A group with a weight that fp32 does not hold is NaN, as one
// with a value that was not finite: as an infinity it would be NaN with a part of an input that is 0, and only there.
__global__ __launch_bounds__(256) void k_lay(const uint8_t* codes, const uint8_t* scales, int32_t out, int32_t in, uint8_t* laid) {
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4, steps = (in + 127) / 128, groups = in / FP4_GROUP;
  const int64_t chunk = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), tile = chunk / steps;
  const int step = (int)(chunk - tile * steps);
  if (tile >= (out + 15) / 16) return;
  const int64_t row = tile * 16 + lr;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = row < out && step * 4 + i < groups ? *(const uint32_t*)(codes + row * (in / 2) + (step * 4 + i) * 16 + lg * 4) : 0u;
  *(uint4*)(laid + chunk * CHUNK + lane * 16) = make_uint4(w[0], w[1], w[2], w[3]);
  uint32_t b = 0;
  if (lg == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) b |= (row < out && step * 4 + i < groups ? scales[row * groups + step * 4 + i] : 127u) << (8 * i);
  b = (uint32_t)__shfl((int)b, lr, 64);    // a row's bytes, to the lanes that have its codes
  uint32_t high = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) high |= (b >> (8 * i) & 255u) - 253u < 2u;
  if (__any(high))
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int nan = beyond(w[i], b >> (8 * i) & 255u);
      nan |= __shfl_xor(nan, 16, 64);
      nan |= __shfl_xor(nan, 32, 64);
      b |= nan ? FP4_NAN << (8 * i) : 0u;
    }
  if (lg == 0) *(uint32_t*)(laid + chunk * CHUNK + 1024 + lr * 4) = b;
}

int refuse_linear(const char* entry, const char* why) {
  thread_local char text[200];
  snprintf(text, sizeof text, "%s: %s", entry, why);
  return dp_set_error(DP_EINVAL, text);
}
const char* why_not_sizes(int32_t out, int32_t in) {
  if (in < FP4_GROUP || in > 1 << 20 || in % FP4_GROUP) return "in must be a multiple of 32 in [32, 2^20]";
  if (out < 1 || out > 1 << 24) return "out must be in [1, 2^24]";
  if ((int64_t)out * in > (int64_t)1 << 36) return "out * in must be at most 2^36";
  return nullptr;
}
const char* why_not_codes(const void* codes, const uint8_t* scales) {
  if (!codes || !scales) return "null pointer";
  return (uintptr_t)codes & 15 ? "codes must be 16-byte aligned" : nullptr;
}
#define REFUSE_IF(expr) do { if (const char* why = (expr)) return refuse_linear(entry, why); } while (0)

}  // namespace

extern "C" size_t dp_fp4_laid_bytes(int32_t out, int32_t in) {
  if (const char* why = why_not_sizes(out, in)) { refuse_linear("dp_fp4_laid_bytes", why); return 0; }
  return (size_t)((out + 15) / 16) * ((in + 127) / 128) * CHUNK;
}

extern "C" int dp_fp4_pack(const void* src, int64_t stride, int32_t out, int32_t in, int32_t dtype, void* codes, uint8_t* scales, void* stream) {
  static const char entry[] = "dp_fp4_pack";
  REFUSE_IF(why_not_sizes(out, in));
  REFUSE_IF(dtype != DP_F32 && dtype != DP_BF16 ? "dtype must be DP_F32 or DP_BF16" : nullptr);
  REFUSE_IF(why_not_codes(codes, scales));
  const int size = dtype == DP_BF16 ? 2 : 4;
  REFUSE_IF(!src ? "null pointer" : nullptr);
  REFUSE_IF((uintptr_t)src & (size - 1) ? "rows must be aligned to their type" : nullptr);
  REFUSE_IF(out > 1 && (stride < 0 || stride > (int64_t)1 << 38) ? "strides must be in [0, 2^38]" : nullptr);
  const hipStream_t st = (hipStream_t)stream;
  const unsigned g = (unsigned)(((int64_t)out * (in / FP4_GROUP) + 255) / 256);
  (void)hipGetLastError();
  if (dtype == DP_BF16) k_pack<bf16_t><<<g, 256, 0, st>>>((const bf16_t*)src, stride, out, in / FP4_GROUP, (uint8_t*)codes, scales);
  else k_pack<float><<<g, 256, 0, st>>>((const float*)src, stride, out, in / FP4_GROUP, (uint8_t*)codes, scales);
  if (hipGetLastError() != hipSuccess) return dp_set_error(DP_EHIP, "dp_fp4_pack: the launch failed");
  return DP_OK;
}

extern "C" int dp_fp4_lay(const void* codes, const uint8_t* scales, int32_t out, int32_t in, void* laid, void* stream) {
  static const char entry[] = "dp_fp4_lay";
  REFUSE_IF(why_not_sizes(out, in));
  REFUSE_IF(why_not_codes(codes, scales));
  REFUSE_IF(!laid ? "null pointer" : nullptr);
  REFUSE_IF((uintptr_t)laid & 63 ? "the laid matrix must be 64-byte aligned" : nullptr);
  const int64_t chunks = (int64_t)((out + 15) / 16) * ((in + 127) / 128);
  (void)hipGetLastError();
  k_lay<<<(unsigned)((chunks + 3) / 4), 256, 0, (hipStream_t)stream>>>((const uint8_t*)codes, scales, out, in, (uint8_t*)laid);
  if (hipGetLastError() != hipSuccess) return dp_set_error(DP_EHIP, "dp_fp4_lay: the launch failed");
  return DP_OK;
}

namespace {
const char* why_not_linear(const dp_fp4_matrix* w, int64_t n) {
  if (!w) return "null pointer";
  if (const char* why = why_not_sizes(w->out, w->in)) return why;
  if (w->dtype != DP_F32 && w->dtype != DP_BF16) return "dtype must be DP_F32 or DP_BF16";
  return n < 0 || n > 1 << 24 || n * w->out > (int64_t)1 << 35 ? "n must be in [0, 2^24], n * out at most 2^35" : nullptr;
}
}  // namespace

extern "C" size_t dp_linear_fp4_workspace_bytes(const dp_fp4_matrix* w, int64_t n) {
  if (const char* why = why_not_linear(w, n)) { refuse_linear("dp_linear_fp4_workspace_bytes", why); return 0; }
  LinearArgs a{};
  a.n = n; a.in = w->in; a.out = w->out;
  return n == 0 ? 0 : partial_bytes(a, w->dtype == DP_BF16 ? route<bf16_t>(a) : route<float>(a));
}

// for the tests, which state the tile that each of their calls is meant to reach: its number, and the ranges of the inputs
extern "C" void dp_linear_fp4_route(const dp_fp4_matrix* w, int64_t n, int32_t* kind_parts) {
  LinearArgs a{};
  a.n = n; a.in = w->in; a.out = w->out;
  const Route r = w->dtype == DP_BF16 ? route<bf16_t>(a) : route<float>(a);
  kind_parts[0] = r.kind;
  kind_parts[1] = r.parts;
}

extern "C" int dp_linear_fp4(const dp_fp4_matrix* w, const void* x, int64_t x_stride, int64_t n, int32_t act, void* y, int64_t y_stride, void* workspace, size_t have, void* stream) {
  static const char entry[] = "dp_linear_fp4";
  REFUSE_IF(why_not_linear(w, n));
  REFUSE_IF(act != DP_ACT_NONE && act != DP_ACT_GELU && act != DP_ACT_SILU ? "act must be DP_ACT_NONE, DP_ACT_GELU or DP_ACT_SILU" : nullptr);
  if (n == 0) return DP_OK;
  const int size = w->dtype == DP_BF16 ? 2 : 4;
  REFUSE_IF(!x || !y || !w->laid ? "null pointer" : nullptr);
  REFUSE_IF((uintptr_t)w->laid & 63 ? "the laid matrix must be 64-byte aligned" : nullptr);
  REFUSE_IF(((uintptr_t)x & 15) || (n > 1 && x_stride % (16 / size)) ? "rows of x must be 16-byte aligned, in their stride too" : nullptr);
  REFUSE_IF(n > 1 && (x_stride < 0 || x_stride > 1 << 21) ? "x_stride must be in [0, 2^21]" : nullptr);
  REFUSE_IF(((uintptr_t)y | (uintptr_t)w->bias) & (size - 1) ? "y and the bias must be aligned to their type" : nullptr);
  REFUSE_IF(n > 1 && (y_stride < w->out || y_stride > (int64_t)1 << 38) ? "y_stride must be in [out, 2^38]" : nullptr);
  REFUSE_IF(x == y ? "y must not be x" : nullptr);
  LinearArgs a{};
  a.laid = (const uint8_t*)w->laid; a.bias = w->bias; a.x = x; a.y = y;
  a.x_s = n > 1 ? x_stride : 0; a.y_s = n > 1 ? y_stride : 0; a.n = n; a.in = w->in; a.out = w->out; a.act = act;
  a.by_four = (uintptr_t)y % (4 * size) == 0 && a.y_s % 4 == 0;
  a.by_eight = (uintptr_t)y % (8 * size) == 0 && a.y_s % 8 == 0 && a.out % 8 == 0;
  const Route r = w->dtype == DP_BF16 ? route<bf16_t>(a) : route<float>(a);
  if (const size_t need = partial_bytes(a, r)) {
    REFUSE_IF((uintptr_t)workspace & 255 ? "the workspace must be 256-byte aligned" : nullptr);
    if (!workspace || have < need) return dp_set_error(DP_ENOMEM, "dp_linear_fp4: workspace too small");
    a.partial = (float*)workspace;
  }
  const hipStream_t st = (hipStream_t)stream;
  (void)hipGetLastError();
  if (w->dtype == DP_BF16) launch<bf16_t>(a, r, st); else launch<float>(a, r, st);
  if (hipGetLastError() != hipSuccess) return dp_set_error(DP_EHIP, "dp_linear_fp4: the launch failed");
  return DP_OK;
}
#undef REFUSE_IF
