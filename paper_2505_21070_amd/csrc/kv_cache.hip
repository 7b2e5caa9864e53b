// Rows of heads on their way into the pages of a key/value cache and out of them: RMSNorm of each head with the 3D rotation
// (dp_qk_norm_rope), the write with or without codes of 8 or 4 bits (dp_kv_write), the two in one pass (dp_kv_write_qkv), the read
// (dp_kv_read).
//
// All are bound by memory: a value is read once and written once, 4 bytes a value in bf16, 3 into codes of 8 bits, 2.5 of 4.  A head's row is 8 to 32 lanes of 16
// bytes, so its sum of squares and its largest value stay within the lanes that hold it, and a channel pair (2i, 2i+1) within one lane.  A wavefront
// takes a run of one token's heads, all queries, all keys or all values: the token's angles are the same for all of them and are computed once, a
// pair a lane, in 64 bits up to the turn's fraction.
#include <math.h>

#include "paged.h"

namespace {

// the rows of a call, queries first, then keys, then values
struct RowArgs {
  const void *q, *k, *v;
  int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs;
  void *qo, *ko;
  int64_t qo_ts, qo_hs, ko_ts, ko_hs;
  void* data;
  uint8_t* scales;
  const int32_t *pos, *slot;
  const void *gq, *gk;
  int64_t n_tokens;
  int32_t hq, hk;
  int32_t runs_q, runs_k, runs;           // runs that a token's queries, its keys (and as well its values), and all of it are cut into
  int32_t per_q, per_k;                   // rows of a run
  int32_t page_shift, n_slots;
  float eps;
  // pair i of an axis with c pairs turns by theta^(-i/c) a step: powers theta^(-2^j/c) of the frame axis (0) and of the other two (1)
  double power[2][6];
};
// where the output of keys and values goes
enum { TO_ROWS = 0, TO_PAGES = 1, TO_CODES = 2, TO_FP4 = 3 };

template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// op over the LANES (8, 16 or 32) lanes of a row, or the 4 or 8 of a group of 32 values, the same in all of them
template <int LANES, typename Op> __device__ __forceinline__ float over_row(float v, Op op) {
  v = op(v, dpp<0xB1>(v));                // quad_perm: lane ^ 1
  v = op(v, dpp<0x4E>(v));                // quad_perm: lane ^ 2
  if constexpr (LANES >= 8) v = op(v, dpp<0x141>(v));    // row_half_mirror: the other quad of 8
  if constexpr (LANES >= 16) v = op(v, dpp<0x140>(v));   // row_mirror: the other half of 16
  if constexpr (LANES >= 32) v = op(v, __shfl_xor(v, 16, 64));
  return v;
}
template <typename T> struct Vec;
template <> struct Vec<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(uint4 u, float (&x)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(uint4 u, float (&x)[4]) {
    x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};

// cos and sin of the token's angles, one pair a lane (a head of 64: lanes 32 .. as lanes 0 ..), handed to the lanes that hold the pairs from pair0 on
template <int HD, int NP>
__device__ __forceinline__ void angles(const RowArgs& a, int64_t t, int lane, int pair0, float (&cs)[NP], float (&sn)[NP]) {
  constexpr int CS = HD / 6, CF = HD / 2 - 2 * CS;          // pairs of the row and column axes, and of the frame axis
  const int32_t pf = a.pos[3 * t], py = a.pos[3 * t + 1], px = a.pos[3 * t + 2];
  const int p = lane & (HD / 2 - 1);
  const bool frame = p < CF;
  const int e = frame ? p : p < CF + CS ? p - CF : p - CF - CS;
  const int32_t at = frame ? pf : p < CF + CS ? py : px;
  double f = 0.15915494309189533577;                         // 1 / (2 pi): angles in turns
#pragma unroll
  for (int j = 0; j < 6; ++j) f *= (e >> j) & 1 ? (frame ? a.power[0][j] : a.power[1][j]) : 1.0;
  const double turns = (double)at * f;
  float c, s;
  sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
#pragma unroll
  for (int i = 0; i < NP; ++i) { cs[i] = __shfl(c, pair0 + i, 64); sn[i] = __shfl(s, pair0 + i, 64); }
}

// The number of a block.  Blocks are handed out to the eight XCDs in turn; with RUNS each XCD gets a run of them, so that tokens that share lines of codes and of
// scale bytes (32 or 128 of them a line) meet in its L2.
template <bool RUNS> __device__ __forceinline__ uint32_t block_of() {
  return RUNS ? (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3) : blockIdx.x;
}

// One wavefront: the rows of a run, 64 / LANES at a time, U of those trips to memory under way at once.  Measured, bf16 heads of 128, 6240 tokens: norm
// of 40 + 40 heads 43 us (256 MB, 5.9 TB/s), 40 + 40 heads into codes of 8 bits 37 us (192 MB, 5.2 TB/s), of 4 bits 31 us (162 MB, 5.3 TB/s; 37 with blocks as they come), 12 + 12 + 12
// with norm into codes of 8 bits 22 us (96 MB, 4.4 TB/s); one token 2.9 us.
template <typename T, int HD, bool NORM, int TO>
__global__ __launch_bounds__(256) void k_head_rows(const RowArgs a) {
  constexpr int N = Vec<T>::N, LANES = HD / N, ROWS = 64 / LANES, U = 4;
  const int lane = threadIdx.x & 63, in_row = lane % LANES, c0 = in_row * N;
  const uint32_t task = block_of<TO == TO_CODES || TO == TO_FP4>() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // below 2^26, see cut()
  const int64_t t = task / (uint32_t)a.runs;
  if (t >= a.n_tokens) return;
  int run = (int)(task % (uint32_t)a.runs);
  // which rows these are; all the same
  const bool is_q = NORM && run < a.runs_q;
  run -= is_q ? 0 : a.runs_q;
  const bool is_v = !is_q && run >= a.runs_k;
  run -= is_v ? a.runs_k : 0;
  const int per = is_q ? a.per_q : a.per_k, of = is_q ? a.hq : a.hk;
  const int first = run * per, last = first + per < of ? first + per : of;
  int32_t slot = 0;
  if constexpr (TO != TO_ROWS) {
    slot = a.slot[t];
    if (!is_q && !(slot >= 0 && slot < a.n_slots)) return;   // a row of padding
  }
  const int64_t hs = is_q ? a.q_hs : is_v ? a.v_hs : a.k_hs;
  const T* const src = (is_q ? (const T*)a.q + t * a.q_ts : is_v ? (const T*)a.v + t * a.v_ts : (const T*)a.k + t * a.k_ts) + c0;
  uint4 raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = first + u * ROWS + lane / LANES;
    raw[u] = r < last ? *(const uint4*)(src + r * hs) : uint4{};
  }
  // y0 = (x0 g0 cos - x1 g1 sin) / rms and y1 = (x0 g0 sin + x1 g1 cos) / rms: the gains are folded into the turn
  float g0c[N / 2], g1s[N / 2], g0s[N / 2], g1c[N / 2];
  if (NORM && !is_v) {
    float g[N], cs[N / 2], sn[N / 2];
    Vec<T>::unpack(*(const uint4*)((const T*)(is_q ? a.gq : a.gk) + c0), g);
    angles<HD, N / 2>(a, t, lane, c0 / 2, cs, sn);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      g0c[i] = g[2 * i] * cs[i]; g0s[i] = g[2 * i] * sn[i];
      g1c[i] = g[2 * i + 1] * cs[i]; g1s[i] = g[2 * i + 1] * sn[i];
    }
  }
  const bool to_rows = TO == TO_ROWS || is_q;
  const int64_t out_hs = is_q ? a.qo_hs : a.ko_hs;
  T* const dst = (is_q ? (T*)a.qo + t * a.qo_ts : (T*)a.ko + t * a.ko_ts) + c0;
  // row 0 of the token's heads in the pages: [page][keys | values][head][token]
  const int64_t row0 = ((((int64_t)(slot >> a.page_shift) * 2 + is_v) * a.hk) << a.page_shift) + (slot & ((1 << a.page_shift) - 1));
  for (int r0 = first; r0 < last; r0 += U * ROWS) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (r0 + u * ROWS >= last) break;
      const int r = r0 + u * ROWS + lane / LANES, next = r + U * ROWS;
      float x[N];
      Vec<T>::unpack(raw[u], x);
      raw[u] = next < last ? *(const uint4*)(src + next * hs) : uint4{};
      if (NORM && !is_v) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) sum = fmaf(x[i], x[i], sum);
        const float inv = rsqrtf(over_row<LANES>(sum, [](float m, float n) { return m + n; }) * (1.f / HD) + a.eps);
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          const float m = x[i] * inv, n = x[i + 1] * inv;
          x[i] = m * g0c[i / 2] - n * g1s[i / 2];
          x[i + 1] = m * g0s[i / 2] + n * g1c[i / 2];
        }
      }
      if (to_rows) {
        if (r < last) *(uint4*)(dst + r * out_hs) = Vec<T>::pack(x);
      } else {
        const int64_t row = row0 + ((int64_t)r << a.page_shift);
        if constexpr (TO == TO_PAGES) {
          if (r < last) *(uint4*)((T*)a.data + row * HD + c0) = Vec<T>::pack(x);
        } else if constexpr (TO == TO_FP4) {
          float top = 0.f;
#pragma unroll
          for (int i = 0; i < N; ++i) top = fmaxf(top, fp4_size(x[i]));
          const uint32_t byte = fp4_byte(over_row<FP4_GROUP / N>(top, [](float m, float n) { return fmaxf(m, n); }));
          const float inv = fp4_inverse(byte);
          if (r < last) {
            uint8_t* const to = (uint8_t*)a.data + row * (HD / 2) + c0 / 2;
            if constexpr (N == 8) *(uint32_t*)to = to_fp4x4(x[0], x[1], x[2], x[3], inv) | to_fp4x4(x[4], x[5], x[6], x[7], inv) << 16;
            else *(uint16_t*)to = (uint16_t)to_fp4x4(x[0], x[1], x[2], x[3], inv);
            if (c0 % FP4_GROUP == 0) a.scales[row * (HD / FP4_GROUP) + c0 / FP4_GROUP] = (uint8_t)byte;
          }
        } else {
          float top = 0.f;
#pragma unroll
          for (int i = 0; i < N; ++i) top = fabsf(x[i]) < INFINITY ? fmaxf(top, fabsf(x[i])) : top;
          const int e = fp8_exponent(over_row<LANES>(top, [](float m, float n) { return fmaxf(m, n); }));
          const float inv = pow2f(-e);
          if (r < last) {
            uint8_t* const to = (uint8_t*)a.data + row * HD + c0;
            if constexpr (N == 8) *(uint2*)to = make_uint2(to_fp8x4(x[0], x[1], x[2], x[3], inv), to_fp8x4(x[4], x[5], x[6], x[7], inv));
            else *(uint32_t*)to = to_fp8x4(x[0], x[1], x[2], x[3], inv);
            if (in_row == 0) a.scales[row] = (uint8_t)(e + 127);
          }
        }
      }
    }
  }
}

// The way back: one row a lane group, keys and values of a token's heads.  40 + 40 heads of 6240 tokens out of codes of 8 bits 29 us (192
// MB, 6.6 TB/s), of 4 bits 27 us (162 MB, 6.0 TB/s), for which eight trips are under way; codes are in the last-level cache after their write.
template <typename T, int HD, int FORMAT>
__global__ __launch_bounds__(256) void k_read_rows(const RowArgs a) {
  constexpr int N = Vec<T>::N, LANES = HD / N, ROWS = 64 / LANES, U = FORMAT == DP_KV_FP4 ? 8 : 4;
  const int lane = threadIdx.x & 63, c0 = lane % LANES * N;
  const uint32_t task = block_of<FORMAT != DP_KV_PLAIN>() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // below 2^26, see cut()
  const int64_t t = task / (uint32_t)a.runs;
  if (t >= a.n_tokens) return;
  int run = (int)(task % (uint32_t)a.runs);
  const bool is_v = run >= a.runs_k;
  run -= is_v ? a.runs_k : 0;
  const int first = run * a.per_k, last = first + a.per_k < a.hk ? first + a.per_k : a.hk;
  const int32_t slot = a.slot[t];
  const bool kept = slot >= 0 && slot < a.n_slots;
  const int64_t page = kept ? slot >> a.page_shift : 0, in_page = kept ? slot & ((1 << a.page_shift) - 1) : 0;
  const int64_t row0 = (((page * 2 + is_v) * a.hk) << a.page_shift) + in_page;
  const int64_t hs = is_v ? a.qo_hs : a.ko_hs;                // the values take the place of the queries
  T* const dst = (is_v ? (T*)a.qo + t * a.qo_ts : (T*)a.ko + t * a.ko_ts) + c0;
  for (int r0 = first; r0 < last; r0 += U * ROWS) {
    typedef typename std::conditional<N == 8, uint2, uint32_t>::type Fp8;
    typedef typename std::conditional<N == 8, uint32_t, uint16_t>::type Fp4;
    typename std::conditional<FORMAT == DP_KV_FP8, Fp8, typename std::conditional<FORMAT == DP_KV_FP4, Fp4, uint4>::type>::type raw[U];
    uint32_t byte[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (FORMAT == DP_KV_FP4 && r0 + u * ROWS >= last) break;
      int r = r0 + u * ROWS + lane / LANES;
      if (r >= last) r = last - 1;
      const int64_t row = row0 + ((int64_t)r << a.page_shift);
      if constexpr (FORMAT == DP_KV_FP8) {
        raw[u] = *(const Fp8*)((const uint8_t*)a.data + row * HD + c0);
        byte[u] = a.scales[row];
      } else if constexpr (FORMAT == DP_KV_FP4) {
        raw[u] = *(const Fp4*)((const uint8_t*)a.data + row * (HD / 2) + c0 / 2);
        byte[u] = a.scales[row * (HD / FP4_GROUP) + c0 / FP4_GROUP];
      } else {
        raw[u] = *(const uint4*)((const T*)a.data + row * HD + c0);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * ROWS + lane / LANES;
      if (r >= last) continue;
      uint4 out;
      if constexpr (FORMAT == DP_KV_PLAIN) out = raw[u];
      else if constexpr (FORMAT == DP_KV_FP4 && N == 8) out = fp4x8_to_bf16(raw[u], __uint_as_float(byte[u] << 23));
      else if constexpr (FORMAT == DP_KV_FP4) { const float4 f = fp4x4_to_f32(raw[u], __uint_as_float(byte[u] << 23)); out = __builtin_bit_cast(uint4, f); }
      else if constexpr (N == 8) out = fp8x8_to_bf16(raw[u], __uint_as_float(byte[u] << 23));
      else { const float4 f = fp8x4_to_f32(raw[u], __uint_as_float(byte[u] << 23)); out = __builtin_bit_cast(uint4, f); }
      if (!kept) out = uint4{};
      *(uint4*)(dst + r * hs) = out;
    }
  }
}

// Runs of heads: as many as give the chip 16384 wavefronts, twice what it holds at the kernels' registers, but none shorter than one of the U
// trips (rows) that a wavefront has under way.
void cut(RowArgs& a, int rows, bool values) {
  const int64_t want = (16384 + a.n_tokens - 1) / a.n_tokens, sections = (a.hq > 0) + 1 + values;
  auto runs = [&](int heads, int32_t& per) -> int32_t {
    if (!heads) return 0;
    int64_t n = (heads + rows - 1) / rows;
    const int64_t most = (want + sections - 1) / sections;
    if (n > most) n = most;
    const int64_t trips = ((heads + n - 1) / n + rows - 1) / rows;
    per = (int32_t)(trips * rows);
    return (heads + per - 1) / per;
  };
  a.runs_q = runs(a.hq, a.per_q);
  a.runs_k = runs(a.hk, a.per_k);
  a.runs = a.runs_q + (values ? 2 : 1) * a.runs_k;
}
unsigned blocks_of(const RowArgs& a) { return (unsigned)((a.n_tokens * a.runs + 31) / 32 * 8); }   // whole eights, see block_of()

void set_powers(RowArgs& a, int hd, float theta) {
  const int cs = hd / 6, cf = hd / 2 - 2 * cs;
  for (int axis = 0; axis < 2; ++axis) {
    a.power[axis][0] = pow((double)theta, -1.0 / (axis ? cs : cf));
    for (int j = 1; j < 6; ++j) a.power[axis][j] = a.power[axis][j - 1] * a.power[axis][j - 1];
  }
}
void set_cache(RowArgs& a, const dp_kv_cache* c) {
  a.data = c->data; a.scales = c->scales;
  a.page_shift = __builtin_ctz((unsigned)c->page_tokens);
  a.n_slots = (int32_t)((int64_t)c->n_pages * c->page_tokens);
  a.hk = c->kv_heads;
}
int to_of(const dp_kv_cache* c) { return c->format == DP_KV_FP4 ? TO_FP4 : c->format == DP_KV_FP8 ? TO_CODES : TO_PAGES; }
#define SET_ROWS(field, rows) do { a.field = (rows)->data; a.field##_ts = (rows)->token_stride; a.field##_hs = (rows)->head_stride; } while (0)

template <typename T, int HD, bool NORM> void launch_to(const RowArgs& a, int to, hipStream_t st) {
  const unsigned g = blocks_of(a);
  if (to == TO_FP4) k_head_rows<T, HD, NORM, TO_FP4><<<g, 256, 0, st>>>(a);
  else if (to == TO_CODES) k_head_rows<T, HD, NORM, TO_CODES><<<g, 256, 0, st>>>(a);
  else if (to == TO_PAGES) k_head_rows<T, HD, NORM, TO_PAGES><<<g, 256, 0, st>>>(a);
  else if constexpr (NORM) k_head_rows<T, HD, NORM, TO_ROWS><<<g, 256, 0, st>>>(a);
}
template <bool NORM> int launch_rows(RowArgs& a, int hd, int dtype, int to, bool values, void* stream, const char* entry) {
  const hipStream_t st = (hipStream_t)stream;
  cut(a, 64 / (hd / (dtype == DP_BF16 ? 8 : 4)), values);
  (void)hipGetLastError();
  if (dtype == DP_BF16) { if (hd == 128) launch_to<bf16_t, 128, NORM>(a, to, st); else launch_to<bf16_t, 64, NORM>(a, to, st); }
  else { if (hd == 128) launch_to<float, 128, NORM>(a, to, st); else launch_to<float, 64, NORM>(a, to, st); }
  if (hipGetLastError() != hipSuccess) { char text[100]; snprintf(text, sizeof text, "%s: the launch failed", entry); return dp_set_error(DP_EHIP, text); }
  return DP_OK;
}
const char* why_not_tokens(int64_t n) { return n < 0 || n > (1 << 24) ? "n_tokens must be in [0, 2^24]" : nullptr; }
const char* why_not_norm(const dp_norm_rope* c) {
  if (!c) return "null pointer";
  if (const char* why = why_not_head(c->q_heads, c->head_dim, c->dtype)) return why;
  if (const char* why = why_not_head(c->kv_heads, c->head_dim, c->dtype)) return why;
  if (!(c->rope_theta >= 1.f && c->rope_theta < INFINITY)) return "rope_theta must be finite and at least 1";
  if (!(c->eps >= 0.f && c->eps < INFINITY)) return "eps must be finite and not negative";
  return nullptr;
}
// what is looked at only if there are tokens
const char* why_not_norm_arrays(const dp_norm_rope* c) {
  if (!c->gq || !c->gk || !c->pos) return "null pointer";
  if (((uintptr_t)c->gq & 15) || ((uintptr_t)c->gk & 15) || ((uintptr_t)c->pos & 3)) return "gains must be 16-byte aligned, positions 4-byte";
  return nullptr;
}
const char* why_not_slots(const int32_t* slot) { return !slot ? "null pointer" : ((uintptr_t)slot & 3) ? "slots must be 4-byte aligned" : nullptr; }

}  // namespace

extern "C" int dp_qk_norm_rope(const dp_norm_rope* c, const dp_rows* q, const dp_rows* k, int64_t n, const dp_rows* qo, const dp_rows* ko, void* stream) {
  static const char entry[] = "dp_qk_norm_rope";
  REFUSE_IF(why_not_norm(c));
  REFUSE_IF(why_not_tokens(n));
  if (n == 0) return DP_OK;
  REFUSE_IF(why_not_norm_arrays(c));
  REFUSE_IF(why_not_rows(q, n, c->q_heads, c->head_dim, c->dtype, false));
  REFUSE_IF(why_not_rows(k, n, c->kv_heads, c->head_dim, c->dtype, false));
  REFUSE_IF(why_not_rows(qo, n, c->q_heads, c->head_dim, c->dtype, true));
  REFUSE_IF(why_not_rows(ko, n, c->kv_heads, c->head_dim, c->dtype, true));
  RowArgs a{};
  SET_ROWS(q, q); SET_ROWS(k, k); SET_ROWS(qo, qo); SET_ROWS(ko, ko);
  a.pos = c->pos; a.gq = c->gq; a.gk = c->gk; a.eps = c->eps; a.n_tokens = n;
  a.hq = c->q_heads; a.hk = c->kv_heads;
  set_powers(a, c->head_dim, c->rope_theta);
  return launch_rows<true>(a, c->head_dim, c->dtype, TO_ROWS, false, stream, entry);
}

extern "C" int dp_kv_write(const dp_kv_cache* c, const dp_rows* k, const dp_rows* v, const int32_t* slot, int64_t n, void* stream) {
  static const char entry[] = "dp_kv_write";
  REFUSE_IF(why_not_cache(c));
  REFUSE_IF(why_not_tokens(n));
  if (n == 0) return DP_OK;
  REFUSE_IF(why_not_slots(slot));
  REFUSE_IF(why_not_rows(k, n, c->kv_heads, c->head_dim, c->dtype, false));
  REFUSE_IF(why_not_rows(v, n, c->kv_heads, c->head_dim, c->dtype, false));
  RowArgs a{};
  SET_ROWS(k, k); SET_ROWS(v, v);
  set_cache(a, c);
  a.slot = slot; a.n_tokens = n;
  return launch_rows<false>(a, c->head_dim, c->dtype, to_of(c), true, stream, entry);
}

extern "C" int dp_kv_write_qkv(const dp_kv_cache* c, const dp_norm_rope* m, const dp_rows* q, const dp_rows* k, const dp_rows* v, const int32_t* slot,
                               int64_t n, const dp_rows* qo, void* stream) {
  static const char entry[] = "dp_kv_write_qkv";
  REFUSE_IF(why_not_cache(c));
  REFUSE_IF(why_not_norm(m));
  REFUSE_IF(m->kv_heads != c->kv_heads || m->head_dim != c->head_dim || m->dtype != c->dtype ? "the norm's kv_heads, head_dim and dtype must be the cache's" : nullptr);
  REFUSE_IF(why_not_tokens(n));
  if (n == 0) return DP_OK;
  REFUSE_IF(why_not_norm_arrays(m));
  REFUSE_IF(why_not_slots(slot));
  REFUSE_IF(why_not_rows(q, n, m->q_heads, c->head_dim, c->dtype, false));
  REFUSE_IF(why_not_rows(k, n, c->kv_heads, c->head_dim, c->dtype, false));
  REFUSE_IF(why_not_rows(v, n, c->kv_heads, c->head_dim, c->dtype, false));
  REFUSE_IF(why_not_rows(qo, n, m->q_heads, c->head_dim, c->dtype, true));
  RowArgs a{};
  SET_ROWS(q, q); SET_ROWS(k, k); SET_ROWS(v, v); SET_ROWS(qo, qo);
  set_cache(a, c);
  a.pos = m->pos; a.gq = m->gq; a.gk = m->gk; a.eps = m->eps; a.slot = slot; a.n_tokens = n;
  a.hq = m->q_heads;
  set_powers(a, c->head_dim, m->rope_theta);
  return launch_rows<true>(a, c->head_dim, c->dtype, to_of(c), true, stream, entry);
}

extern "C" int dp_kv_read(const dp_kv_cache* c, const int32_t* slot, int64_t n, const dp_rows* ko, const dp_rows* vo, void* stream) {
  static const char entry[] = "dp_kv_read";
  REFUSE_IF(why_not_cache(c));
  REFUSE_IF(why_not_tokens(n));
  if (n == 0) return DP_OK;
  REFUSE_IF(why_not_slots(slot));
  REFUSE_IF(why_not_rows(ko, n, c->kv_heads, c->head_dim, c->dtype, true));
  REFUSE_IF(why_not_rows(vo, n, c->kv_heads, c->head_dim, c->dtype, true));
  RowArgs a{};
  set_cache(a, c);
  SET_ROWS(ko, ko);
  SET_ROWS(qo, vo);
  a.slot = slot; a.n_tokens = n;
  const hipStream_t st = (hipStream_t)stream;
  cut(a, 64 / (c->head_dim / (c->dtype == DP_BF16 ? 8 : 4)), true);
  const unsigned g = blocks_of(a);
  (void)hipGetLastError();
#define READ(T, HD) do { if (c->format == DP_KV_FP4) k_read_rows<T, HD, DP_KV_FP4><<<g, 256, 0, st>>>(a); \
    else if (c->format == DP_KV_FP8) k_read_rows<T, HD, DP_KV_FP8><<<g, 256, 0, st>>>(a); else k_read_rows<T, HD, DP_KV_PLAIN><<<g, 256, 0, st>>>(a); } while (0)
  if (c->dtype == DP_BF16) { if (c->head_dim == 128) READ(bf16_t, 128); else READ(bf16_t, 64); }
  else { if (c->head_dim == 128) READ(float, 128); else READ(float, 64); }
#undef READ
  if (hipGetLastError() != hipSuccess) return dp_set_error(DP_EHIP, "dp_kv_read: the launch failed");
  return DP_OK;
}
