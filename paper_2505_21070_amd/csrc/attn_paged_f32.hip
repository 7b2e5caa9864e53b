// Attention of new tokens over the pages of a key/value cache, fp32 (dp_attn_paged).
//
// As in bf16 (attn_paged_bf16.hip), on v_mfma_f32_16x16x4_f32: S^T = K Q^T, whose accumulators, once turned into weights, are the B operand of O^T = V^T P^T
// register by register (register r of a lane is key (lane >> 4) * 4 + r, and step r of the second product takes just those four keys).  The
// head dim's order in the first product is free: a lane takes 16 bytes of a key's or query's row and uses their four values in four steps.
// LDS rows are padded by 16 bytes: 16 rows of 16 bytes, and four rows of 64, four apart, spread over the 64 banks.
// The matrix pipe does 1/16 of bf16's rate, so everything else hides behind it.
#include <math.h>

#include "attn_paged.h"

namespace {

__device__ __forceinline__ f32x4 mfma(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// A tile of TK keys and values on its way from the pages into LDS, in the registers of W wavefronts, of which this is number w: four
// channels a lane and trip.
template <int HD, int TK, int W, bool CODES> struct Carry {
  static constexpr int LANES = HD / 4, RW = 64 / LANES, N = TK / (W * RW);   // lanes of a row, rows of a trip of one wavefront, trips
  static_assert(N * W * RW == TK && RW <= 16, "a trip's rows lie in one page");
  typedef typename std::conditional<CODES, uint32_t, f32x4>::type Raw;
  Raw raw[N];
  uint32_t byte[CODES ? N : 1];
  __device__ __forceinline__ void load(const PagedArgs& a, const Block& b, int key0, int64_t to_values, int w, int lane) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t row = page_row(a, b, key0 + (i * W + w) * RW) + to_values;
      raw[i] = *(const Raw*)((const char*)a.data + row * (HD * (CODES ? 1 : 4)) + lane * sizeof(Raw));
      if constexpr (CODES) byte[i] = (a.scales + row)[lane / LANES];
    }
  }
  __device__ __forceinline__ void store(float* tile, int w, int lane) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float* const at = tile + ((i * W + w) * RW + lane / LANES) * (HD + 4) + lane % LANES * 4;
      if constexpr (CODES) *(float4*)at = fp8x4_to_f32(raw[i], __uint_as_float(byte[i] << 23));
      else *(f32x4*)at = raw[i];
    }
  }
};

// One tile of KT * 16 keys: scores, what a row does not see, the online softmax, the weighted sum.
template <int HD, int KT, int NT>
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
#pragma unroll
  for (int c = 0; c < HD / 16; c += 2) {
    f32x4 k[2][KT];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) k[h][kt] = *(const f32x4*)(ktile + (kt * 16 + lr) * RS + (c + h) * 16 + lg * 4);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          sc[t][kt] = mfma(k[0][kt][j], qf[t][c][j], sc[t][kt]);
          odd[t][kt] = mfma(k[1][kt][j], qf[t][c + 1][j], odd[t][kt]);
        }
  }
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
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) o[d][t] *= alpha;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[t][kt][r] = __builtin_amdgcn_exp2f(fmaf(sc[t][kt][r], a.scale, -ref));
        z[t].l += p[t][kt][r];
      }
  }
  if (!border) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) {
          const float v = vtile[(kt * 16 + lg * 4 + r) * RS + d * 16 + lr];
#pragma unroll
          for (int t = 0; t < NT; ++t) o[d][t] = mfma(v, p[t][kt][r], o[d][t]);
        }
    return;
  }
  // A value that is not finite must not meet the weight 0 of a row that does not see its key (0 * infinity is NaN): it is multiplied as 0, and rows that do
  // see +inf, -inf or NaN are found by products of ones and get it added.
#pragma unroll
  for (int d = 0; d < HD / 16; ++d) {
    float v[KT][4];
    bool bad = false;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        v[kt][r] = vtile[(kt * 16 + lg * 4 + r) * RS + d * 16 + lr];
        bad |= !(fabsf(v[kt][r]) < INFINITY);
      }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) o[d][t] = mfma(fabsf(v[kt][r]) < INFINITY ? v[kt][r] : 0.f, p[t][kt][r], o[d][t]);
    if (!__any(bad)) continue;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4 np{0.f, 0.f, 0.f, 0.f}, nn = np, nx = np;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float x = v[kt][r], one = sc[t][kt][r] == -INFINITY ? 0.f : 1.f;
          np = mfma(x == INFINITY ? 1.f : 0.f, one, np);
          nn = mfma(x == -INFINITY ? 1.f : 0.f, one, nn);
          nx = mfma(x != x ? 1.f : 0.f, one, nx);
        }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = o[d][t][r] + (np[r] > 0.f ? INFINITY : 0.f) - (nn[r] > 0.f ? INFINITY : 0.f);
        o[d][t][r] = nx[r] > 0.f ? __uint_as_float(0x7fc00000u) : x;
      }
    }
  }
}

// Four wavefronts.  QG = 4: each has NT * 16 rows of its own, and they share tiles of 32 keys.  QG = 1: all have the same NT * 16 rows and deal the keys
// out in tiles of 16 (wavefront w: tiles w, w + 4, ...), and meet in LDS at the end.  Either way the next tile is on its way in registers.
template <int HD, int NT, int QG, bool CODES>
__global__ __launch_bounds__(256) void k_paged_f32(const PagedArgs a) {
  constexpr int KG = 4 / QG, TK = QG == 1 ? 16 : 32, KT = TK / 16, RS = HD + 4, QB = QG * NT * 16, TILE = TK * RS;
  constexpr int JOIN = QG == 1 ? 4 * 16 * 2 + 4 * 16 * RS : 0, SIZE = KG * 2 * TILE;
  __shared__ __align__(16) float smem[SIZE > JOIN ? SIZE : JOIN];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), qt = wave % QG, kg = wave / QG;
  Walk<QB, KG * TK, false> walk(a, blockIdx.x);
  Piece p;
  if (!walk.next(a, p)) return;
  const Block& b = p.b;
  const int k0 = p.k0, k1 = p.k1;
  f32x4 qf[NT][HD / 16], o[HD / 16][NT];
  int end[NT];
  Soft z[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = b.first + (qt * NT + t) * 16 + (lane & 15);
    const float* const q = (const float*)a.q + row_at(a, b, row < b.rows ? row : b.rows - 1, a.q_ts, a.q_hs) + (lane >> 4) * 4;
#pragma unroll
    for (int c = 0; c < HD / 16; ++c) qf[t][c] = *(const f32x4*)(q + c * 16);
    end[t] = row_end(a, b, row);
    z[t] = Soft{-INFINITY, 0.f};
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) o[d][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  float* const kt = smem + kg * 2 * TILE;
  float* const vt = kt + TILE;
  const int64_t to_values = (int64_t)a.hk << a.page_shift;
  Carry<HD, TK, QG, CODES> ck, cv;
  int key = k0 + kg * TK;
  if (key < k1) { ck.load(a, b, key, 0, qt, lane); cv.load(a, b, key, to_values, qt, lane); }
  const bool gaps = __builtin_amdgcn_readfirstlane((int)pages_missing(a, b, k0, k1));
  for (; key < k1; key += KG * TK) {
    if constexpr (QG > 1) __syncthreads();
    ck.store(kt, qt, lane);
    cv.store(vt, qt, lane);
    if constexpr (QG > 1) __syncthreads();
    if (key + KG * TK < k1) { ck.load(a, b, key + KG * TK, 0, qt, lane); cv.load(a, b, key + KG * TK, to_values, qt, lane); }
    step<HD, KT, NT>(a, b, kt, vt, qf, key, key + TK > b.whole || gaps, end, gaps, z, o, lane);
  }
  if constexpr (QG > 1) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int row = (qt * NT + t) * 16 + (lane & 15);
      const float l = over_lanes(z[t].l);
      if (b.first + row >= b.rows) continue;
      if (p.slot < 0) {
        float* const out = (float*)a.out + row_at(a, b, b.first + row, a.o_ts, a.o_hs) + (lane >> 4) * 4;
        const float inv = inverse(l);
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) *(f32x4*)(out + d * 16) = o[d][t] * inv;
      } else {
        float* const ps = a.partial + (size_t)p.slot * (QB * (2 + HD));
        if (lane < 16) { ps[row] = z[t].m; ps[QB + row] = l; }
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) *(f32x4*)(ps + 2 * QB + row * HD + d * 16 + (lane >> 4) * 4) = o[d][t];
      }
    }
  } else {
    join_waves<float, HD, NT, 4>(a, b, smem, z, o, p.slot, wave, lane);
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
    static const Kind wide[2] = {{64, 512, 32, 370, 200, 800}, {128, 512, 32, 720, 380, 800}}, narrow[2] = {{64, 512, 32, 190, 110, 800}, {128, 512, 32, 370, 200, 800}};
    choose(a, head_dim == 128 ? wide : narrow, rows <= 64 ? 1 : 2, head_dim, r);
  }
  r.tiles_of_seq = (rows + r.qb - 1) / r.qb;
  return r;
}
template <int HD, int NT, int QG> void launch(const PagedArgs& a, bool codes, hipStream_t st) {
  constexpr int QB = QG * NT * 16;
  const int64_t blocks = (int64_t)a.tiles * a.hk;
  const unsigned g = (unsigned)(blocks * a.parts);
  if (codes) k_paged_f32<HD, NT, QG, true><<<g, 256, 0, st>>>(a); else k_paged_f32<HD, NT, QG, false><<<g, 256, 0, st>>>(a);
  if (a.parts > 1) k_paged_join<float, HD, QB><<<(unsigned)(blocks * QB * (HD / 4) / 256), 256, 0, st>>>(a);
}
template <int HD> void launch(const PagedArgs& a, int qb, bool codes, hipStream_t st) {
  if (qb == 16) launch<HD, 1, 1>(a, codes, st);
  else if (qb == 64) launch<HD, 1, 4>(a, codes, st);
  else launch<HD, 2, 4>(a, codes, st);
}

}  // namespace

size_t launch_attn_paged_f32(PagedArgs a, int head_dim, bool codes, bool go, hipStream_t st) {
  const Route r = route(a, head_dim);
  a.tiles = (int32_t)r.tiles; a.tiles_of_seq = (int32_t)r.tiles_of_seq; a.parts = r.parts; a.part_keys = r.part_keys;
  if (go) { if (head_dim == 128) launch<128>(a, r.qb, codes, st); else launch<64>(a, r.qb, codes, st); }
  return r.parts > 1 ? (size_t)r.tiles * a.hk * r.parts * ((size_t)r.qb * (2 + head_dim) * sizeof(float)) : 0;
}
