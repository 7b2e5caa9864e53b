// Attention of new tokens over the pages of a key/value cache, fp32 (dp_attn_paged).
//
// As in bf16 (attn_paged_bf16.hip), on v_mfma_f32_16x16x4_f32: S^T = K Q^T, whose accumulators, once turned into weights, are the B operand of O^T = V^T P^T
// register by register (register r of a lane is key (lane >> 4) * 4 + r, and step r of the second product takes just those four keys).  The
// head dim's order in the first product is free: a lane takes 16 bytes of a key's or query's row and uses their four values in four steps.
// LDS rows are padded by 16 bytes, so that 16 rows of 16 bytes spread over the 64 banks.  The order of O^T's rows is free as well: a lane reads its
// channels of a value's row with 16-byte reads.
// The matrix pipe does 1/16 of bf16's rate, so everything else hides behind it: 4096 x 4096 x 16 heads of 128 1156 us, 119 TFLOP/s, of 64 590 us, 116; one
// token's rows are bound by memory: 64 sequences of 2000 keys, 8 heads of 128, 187 us, 5.6 TB/s.  Codes go through the same instructions and save memory alone, of which a lane asks for 4 (8 bits) or 2 bytes (4
// bits) at once: the same 64 sequences 107 and 115 us; one token of 64 sequences of 100 .. 16000 keys, 32 heads on 8, 590 and 704; 1560 x 20280 x 12 heads 1.71 and 1.75 ms, as they are 1.68.
#include <math.h>

#include "attn_paged.h"

namespace {

__device__ __forceinline__ f32x4 mfma(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// A tile of TK keys and values on its way from the pages into LDS, in the registers of W wavefronts, of which this is number w: four
// channels a lane and trip.
template <int HD, int TK, int W, int FORMAT> struct Carry {
  static constexpr bool CODES = FORMAT != DP_KV_PLAIN;
  static constexpr int ROW = FORMAT == DP_KV_FP4 ? HD / 2 : FORMAT == DP_KV_FP8 ? HD : HD * 4;   // bytes of a row in the pages
  static constexpr int LANES = HD / 4, RW = 64 / LANES, N = TK / (W * RW);   // lanes of a row, rows of a trip of one wavefront, trips
  static_assert(N * W * RW == TK && RW <= 16, "a trip's rows lie in one page");
  typedef typename std::conditional<FORMAT == DP_KV_FP4, uint16_t, typename std::conditional<CODES, uint32_t, f32x4>::type>::type Raw;
  Raw raw[N];
  uint32_t byte[CODES ? N : 1];
  typedef TileRows<N, W, RW> Rows;
  __device__ __forceinline__ void load(const PagedArgs& a, const Rows& rows, int64_t to_values, int w, int lane) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t row = rows.row(i, w) + to_values;
      raw[i] = *(const Raw*)((const char*)a.data + row * ROW + lane * sizeof(Raw));
      if constexpr (FORMAT == DP_KV_FP4) byte[i] = (a.scales + row * (HD / FP4_GROUP))[lane / (FP4_GROUP / 4)];
      else if constexpr (CODES) byte[i] = (a.scales + row)[lane / LANES];
    }
  }
  __device__ __forceinline__ void store(float* tile, int w, int lane) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float* const at = tile + ((i * W + w) * RW + lane / LANES) * (HD + 4) + lane % LANES * 4;
      if constexpr (FORMAT == DP_KV_FP4) *(float4*)at = fp4x4_to_f32(raw[i], __uint_as_float(byte[i] << 23));
      else if constexpr (CODES) *(float4*)at = fp8x4_to_f32(raw[i], __uint_as_float(byte[i] << 23));
      else *(f32x4*)at = raw[i];
    }
  }
};

// One tile of KT * 16 keys: scores, what a row does not see (border), the online softmax, the weighted sum (at a border and CAREFUL: with values
// looked at; CAREFUL: and sums that are not finite kept).
template <int HD, int KT, int NT, bool CAREFUL>
__device__ __forceinline__ void step(const PagedArgs& a, const Block& b, const float* ktile, const float* vtile, const f32x4 (&qf)[NT][HD / 16], int key0,
                                     bool border, const int (&end)[NT], bool gaps, Soft (&z)[NT], f32x4 (&o)[HD / 16][NT], int lane) {
  constexpr int RS = HD + 4;
  const int lr = lane & 15, lg = lane >> 4;
  // two chains of sums for each tile of scores, so that no product waits for the one before it
  f32x4 sc[NT][KT], odd[NT][KT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) sc[t][kt] = odd[t][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
  // operands are read from LDS a batch of products before they are used
  f32x4 k[2][2][KT];
  auto read_k = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) k[(c / 2) & 1][h][kt] = *(const f32x4*)(ktile + (kt * 16 + lr) * RS + (c + h) * 16 + lg * 4);
  };
  read_k(0);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int c = 0; c < HD / 16; c += 2) {
    if (c + 2 < HD / 16) read_k(c + 2);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          sc[t][kt] = mfma(k[(c / 2) & 1][0][kt][j], qf[t][c][j], sc[t][kt]);
          odd[t][kt] = mfma(k[(c / 2) & 1][1][kt][j], qf[t][c + 1][j], odd[t][kt]);
        }
    __builtin_amdgcn_sched_barrier(0);
  }
  // the values of this lane's first key: row n of channel tile d is channel n * (HD / 16) + d, so that a lane's channels lie together
  float v[2][HD / 16];
  auto read_v = [&](int i) __attribute__((always_inline)) {            // key (i / 4) * 16 + lg * 4 + i % 4
    const float* const at = vtile + ((i >> 2) * 16 + lg * 4 + (i & 3)) * RS + lr * (HD / 16);
#pragma unroll
    for (int d = 0; d < HD / 16; d += 4) {
      const f32x4 x = *(const f32x4*)(at + d);
      v[i & 1][d] = x[0]; v[i & 1][d + 1] = x[1]; v[i & 1][d + 2] = x[2]; v[i & 1][d + 3] = x[3];
    }
  };
  read_v(0);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) sc[t][kt] += odd[t][kt];
  const uint32_t gone = gaps ? missing<KT>(a, b, key0, lane) : 0;
  f32x4 p[NT][KT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (border) hide<KT>(sc[t], key0, end[t], gone, lane);
    float ref;
    const float alpha = raise(z[t], maximum<KT>(sc[t], KT) * a.scale, ref);
    if (CAREFUL && __any(alpha == 0.f)) {
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) o[d][t] = lowered(o[d][t], alpha);
    } else {
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) o[d][t] *= alpha;
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[t][kt][r] = __builtin_amdgcn_exp2f(fmaf(sc[t][kt][r], a.scale, -ref));
        z[t].l += p[t][kt][r];
      }
  }
  // A value that is not finite must not meet the weight 0 of a row that does not see its key (0 * infinity is NaN): at a border it is multiplied as 0, and rows
  // that do see +inf, -inf or NaN are found by products of ones and get it added.
#pragma unroll
  for (int i = 0; i < KT * 4; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    if (i + 1 < KT * 4) read_v(i + 1);
    __builtin_amdgcn_sched_barrier(0);
    bool bad = false;
    float x[HD / 16];
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) x[d] = v[i & 1][d];
    if (border || CAREFUL) {
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) bad |= !(fabsf(x[d]) < INFINITY);
    }
    if ((border || CAREFUL) && __any(bad)) {
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const f32x4 zero{0.f, 0.f, 0.f, 0.f};
          const float one = sc[t][i >> 2][i & 3] == -INFINITY ? 0.f : 1.f;
          const f32x4 np = mfma(x[d] == INFINITY ? 1.f : 0.f, one, zero), nn = mfma(x[d] == -INFINITY ? 1.f : 0.f, one, zero), nx = mfma(x[d] != x[d] ? 1.f : 0.f, one, zero);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float y = o[d][t][r] + (np[r] > 0.f ? INFINITY : 0.f) - (nn[r] > 0.f ? INFINITY : 0.f);
            o[d][t][r] = nx[r] > 0.f ? __uint_as_float(0x7fc00000u) : y;
          }
        }
        x[d] = fabsf(x[d]) < INFINITY ? x[d] : 0.f;
      }
    }
#pragma unroll
    for (int d = 0; d < HD / 16; ++d)
#pragma unroll
      for (int t = 0; t < NT; ++t) o[d][t] = mfma(x[d], p[t][i >> 2][i & 3], o[d][t]);
  }
}

// Four wavefronts.  QG = 4: each has 16 rows of its own, and they share tiles of 32 keys.  QG = 1: all have the same 16 rows and deal the keys
// out in tiles of 16 (wavefront w: tiles w, w + 4, ...), and meet in LDS at the end.  Either way the next tile is on its way in registers.  Registers are bounded for
// three blocks on a CU (heads of 64: four): 4096 x 4096 x 16 heads 1242 -> 1148 us.
template <int HD, int QG, int FORMAT>
__global__ __launch_bounds__(256, QG == 4 ? (HD == 64 ? 4 : 3) : 2) void k_paged_f32(const PagedArgs a) {
  constexpr int NT = 1, KG = 4 / QG, TK = QG == 1 ? 16 : 32, KT = TK / 16, RS = HD + 4, QB = QG * NT * 16, TILE = TK * RS;
  constexpr int JOIN = QG == 1 ? 4 * 16 * 2 + 4 * 16 * RS : 0, SIZE = KG * 2 * TILE;
  __shared__ __align__(16) float smem[SIZE > JOIN ? SIZE : JOIN];
  __shared__ int again;                                      // whether a wavefront has sums that are not finite
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), qt = wave % QG, kg = wave / QG;
  Walk<QB, KG * TK, false> walk(a, blockIdx.x);
  Piece p;
  if (!walk.next(a, p)) return;
  const Block& b = p.b;
  const int k0 = p.k0, k1 = p.k1;
  f32x4 qf[NT][HD / 16], o[HD / 16][NT];
  int end[NT];
  Soft z[NT];
  float* const kt = smem + kg * 2 * TILE;
  float* const vt = kt + TILE;
  const int64_t to_values = (int64_t)a.hk << a.page_shift;
  Carry<HD, TK, QG, FORMAT> ck, cv;
  auto load = [&](int at, int lane) __attribute__((always_inline)) {
    typename decltype(ck)::Rows rows;
    rows.look(a, b, at, qt);
    ck.load(a, rows, 0, qt, lane);
    cv.load(a, rows, to_values, qt, lane);
  };
  const int first = k0 + kg * TK;
  if (first < k1) load(first, lane);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = b.first + (qt * NT + t) * 16 + (lane & 15);
    const float* const q = (const float*)a.q + row_at(a, b, row < b.rows ? row : b.rows - 1, a.q_ts, a.q_hs) + (lane >> 4) * 4;
#pragma unroll
    for (int c = 0; c < HD / 16; ++c) qf[t][c] = *(const f32x4*)(q + c * 16);
    end[t] = row_end(a, b, row);
  }
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      z[t] = Soft{-INFINITY, 0.f};
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) o[d][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  clear();
  if (threadIdx.x == 0) again = 0;                           // seen by all behind the look at the pages
  const bool gaps = __builtin_amdgcn_readfirstlane((int)pages_missing(a, b, k0, k1));
  auto put = [&](int lane) __attribute__((always_inline)) {
    if constexpr (QG > 1) __syncthreads();
    ck.store(kt, qt, lane);
    cv.store(vt, qt, lane);
    if constexpr (QG > 1) __syncthreads();
  };
  for (int key = first; key < k1; key += KG * TK) {
    put(lane);
    if (key + KG * TK < k1) load(key + KG * TK, lane);
    step<HD, KT, NT, false>(a, b, kt, vt, qf, key, key + TK > b.whole || gaps, end, gaps, z, o, lane);
  }
  bool careful = !__all(finite(o));
  if constexpr (QG > 1) {
    if (careful) again = 1;
    __syncthreads();
    careful = again;
  }
  if (__builtin_expect(careful, 0)) {
    clear();
    for (int key = first; key < k1; key += KG * TK) {
      const int lane = fresh_lane();
      load(key, lane);
      put(lane);
      step<HD, KT, NT, true>(a, b, kt, vt, qf, key, key + TK > b.whole || gaps, end, gaps, z, o, lane);
    }
  }
  if constexpr (QG > 1) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int row = (qt * NT + t) * 16 + (lane & 15);
      const float l = over_lanes(z[t].l);
      if (b.first + row >= b.rows) continue;
      if (p.slot < 0) {
        put_row<HD, NT, true>((float*)a.out + row_at(a, b, b.first + row, a.o_ts, a.o_hs), o, t, lane >> 4, inverse(l));
      } else {
        float* const ps = a.partial + (size_t)p.slot * (QB * (2 + HD));
        if (lane < 16) { ps[row] = z[t].m; ps[QB + row] = l; }
        put_row<HD, NT, true>(ps + 2 * QB + row * HD, o, t, lane >> 4, 1.f);
      }
    }
  } else {
    join_waves<float, HD, NT, 4, true>(a, b, smem, z, o, p.slot, wave, lane);
  }
}

Route route(const PagedArgs& a, int head_dim) {
  Route r{};
  const int64_t rows = (int64_t)a.max_q * a.shared, keys = a.max_kv;          // of a sequence, at most
  if (rows <= 16) {
    r.qb = 16;
    r.tiles = tiles_of_call(a, 16);
    // ranges for four times as many blocks as there are CUs, none shorter than two trips of the four wavefronts
    const int64_t blocks = r.tiles * a.hk;
    int64_t parts = (1024 + blocks - 1) / blocks;
    if (parts > (keys + 127) / 128) parts = (keys + 127) / 128;
    if (parts > 256) parts = 256;
    if (parts < 1) parts = 1;
    r.part_keys = (int)(((keys + parts - 1) / parts + 63) / 64 * 64);
    r.parts = r.part_keys > 0 ? (int)((keys + r.part_keys - 1) / r.part_keys) : 1;
    if (r.parts < 1) r.parts = 1;
  } else {
    // Measured: a step of 32 keys takes 2.8, 4.8 and 7.0 us with one, two and three blocks on a CU (heads of 64: 1.6, 2.6, 3.8 and 4.9).  Blocks of 128 rows (two
    // columns a wavefront) are no faster at any size.
    static const Kind wide{64, 32, 4, 3, 3, {279, 484, 703}, 800}, narrow{64, 32, 4, 4, 4, {158, 260, 377, 492}, 800};
    choose(a, head_dim == 128 ? &wide : &narrow, 1, head_dim, r);
  }
  r.tiles_of_seq = (rows + r.qb - 1) / r.qb;
  return r;
}
template <int HD, int QG> void launch(const PagedArgs& a, int format, hipStream_t st) {
  constexpr int QB = QG * 16;
  const int64_t blocks = (int64_t)a.tiles * a.hk;
  const unsigned g = (unsigned)(blocks * a.parts);
  if (format == DP_KV_FP4) k_paged_f32<HD, QG, DP_KV_FP4><<<g, 256, 0, st>>>(a);
  else if (format == DP_KV_FP8) k_paged_f32<HD, QG, DP_KV_FP8><<<g, 256, 0, st>>>(a);
  else k_paged_f32<HD, QG, DP_KV_PLAIN><<<g, 256, 0, st>>>(a);
  launch_join<float, HD, QB>(a, st);
}
template <int HD> void launch(const PagedArgs& a, int qb, int format, hipStream_t st) {
  if (qb == 16) launch<HD, 1>(a, format, st); else launch<HD, 4>(a, format, st);
}

}  // namespace

Route route_attn_paged_f32(const PagedArgs& a, int head_dim) { return route(a, head_dim); }
void launch_attn_paged_f32(const PagedArgs& a, const Route& r, int head_dim, int format, hipStream_t st) {
  if (head_dim == 128) launch<128>(a, r.qb, format, st); else launch<64>(a, r.qb, format, st);
}
