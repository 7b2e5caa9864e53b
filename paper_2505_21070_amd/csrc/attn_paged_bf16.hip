// Attention of new tokens over the pages of a key/value cache, bf16 (dp_attn_paged).
//
// Scores are computed transposed, S^T = K Q^T (v_mfma_f32_16x16x32_bf16), so that a lane's accumulators belong to one row and, turned
// into weights and rounded to bf16, are the B operand of O^T = V^T P^T as they stand.  The rows of a block are (new token, query head)
// pairs that share a key head: the matrix instructions' columns are filled by shared heads as by tokens, and one read of the keys serves
// all of them.  Keys and values go from their pages into LDS in rows as they lie in the page, through registers (codes of 8 or 4 bits become bf16 on the way,
// exactly) or, whole tiles of blocks of many rows that are held as they are, by direct loads; the operand V^T comes out of LDS by transposing reads (ds_read_b64_tr_b16), whose four consecutive keys a lane are just
// those of four accumulators.
//
// A tile of keys is either seen whole by every row of the block, or holds a border (the sequence's end, a causal border, a page that
// does not exist).  Whole tiles come first; a tile with a border is masked key by key, and its values that are not finite are kept from
// the rows that do not see them (weighted_sum_checked).
#include <math.h>

#include <atomic>

#include "attn_paged.h"
#include "kernels.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float add_pk(uint32_t pk, float acc) {          // acc + lo + hi of a packed bf16 pair
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk), __builtin_bit_cast(bf16x2, 0x3f803f80u), acc, false);
}
__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// LDS by byte address: 16 bytes in and out, and the transposing read of 8
__device__ __forceinline__ uint32_t lds_address(const void* p) {
#ifdef __HIP_DEVICE_COMPILE__
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
#else
  return 0;
#endif
}
// an address that the constants added to it stay apart from, in the instructions' offset fields
__device__ __forceinline__ uint32_t lds_base(uint32_t at) {
#ifdef __HIP_DEVICE_COMPILE__
  asm("" : "+v"(at));
#endif
  return at;
}
__device__ __forceinline__ bf16x8 lds_get(uint32_t at) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_bit_cast(bf16x8, *(const __attribute__((address_space(3))) u32x4*)at);
#else
  return bf16x8{};
#endif
}
template <typename V> __device__ __forceinline__ void lds_put(uint32_t at, V v) {
#ifdef __HIP_DEVICE_COMPILE__
  *(__attribute__((address_space(3))) V*)at = v;
#endif
}
__device__ __forceinline__ bf16x4 lds_get_transposed(uint32_t at) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)at));
#else
  return bf16x4{};
#endif
}

// LDS tiles: rows of HD bf16 values, their 16-byte chunks exchanged by the row so that what an instruction reads spreads over the 64
// banks: 16 rows of one chunk column (keys, 16 bytes a lane) and 16 rows of two (values, the transposing read's 32 bytes of a row).
template <int HD> __device__ __forceinline__ int k_swizzle(int row) { return HD == 128 ? row & 15 : (row >> 1) & 7; }
template <int HD> __device__ __forceinline__ int v_swizzle(int row) { return HD == 128 ? (row & 7) << 1 : ((row >> 1) & 3) << 1; }

// A tile of TK keys and values on its way from the pages into LDS, in the registers of W wavefronts, of which this is number w.
template <int HD, int TK, int W, int FORMAT> struct Carry {
  static constexpr bool CODES = FORMAT != DP_KV_PLAIN;
  static constexpr int ROW = FORMAT == DP_KV_FP4 ? HD / 2 : CODES ? HD : HD * 2;   // bytes of a row in the pages
  static constexpr int MOST = ROW / 4 < 16 ? ROW / 4 : 16;                   // a trip has 16 rows at most
  static constexpr int LB = TK * ROW / (W * 64) < MOST ? TK * ROW / (W * 64) : MOST;   // bytes a lane takes at once
  static constexpr int WIDER = FORMAT == DP_KV_FP4 ? 4 : CODES ? 2 : 1;      // bytes in LDS for one in the pages
  static constexpr int N = TK * ROW / (W * 64 * LB), RW = 64 * LB / ROW;     // trips, rows of a trip of one wavefront
  static_assert(N * W * RW == TK && RW <= 16 && (LB == 16 || LB == 8), "a trip's rows lie in one page");
  typedef typename std::conditional<LB == 16, u32x4, u32x2>::type Raw;
  Raw raw[N];
  uint32_t byte[CODES ? N : 1];
  // where the trips' rows lie in the pages, for keys key0 .. of the block's sequence: uniform
  typedef TileRows<N, W, RW> Rows;
  static __device__ __forceinline__ Rows rows(const PagedArgs& a, const Block& b, int key0, int w) {
    Rows r;
    r.look(a, b, key0, w);
    return r;
  }
  // to_values: rows between a head's keys and its values
  __device__ __forceinline__ void load(const PagedArgs& a, const Rows& rows, int64_t to_values, int w, int lane) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t row = rows.row(i, w) + to_values;
      raw[i] = *(const Raw*)((const char*)a.data + row * ROW + lane * LB);
      if constexpr (FORMAT == DP_KV_FP4) byte[i] = (a.scales + row * (HD / FP4_GROUP))[lane * LB / (FP4_GROUP / 2)];
      else if constexpr (CODES) byte[i] = (a.scales + row)[lane / (ROW / LB)];
    }
  }
  template <bool VALUES> __device__ __forceinline__ void store(uint32_t tile, int w, int lane) const {
    // rows of a trip differ from the first trip's in higher bits, and the exchange takes each bit by itself: few addresses, the rest in the instructions' offsets
    const int row = w * RW + lane / (ROW / LB);
    const uint32_t in_row = lane % (ROW / LB) * LB * WIDER ^ (VALUES ? v_swizzle<HD>(row) : k_swizzle<HD>(row)) * 16, at = tile + row * HD * 2;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t x = (VALUES ? v_swizzle<HD>(i * W * RW) : k_swizzle<HD>(i * W * RW)) * 16, off = i * W * RW * HD * 2;
      if constexpr (!CODES) {
        lds_put(lds_base((in_row ^ x) + at) + off, raw[i]);
      } else if constexpr (FORMAT == DP_KV_FP4) {
        const float f = __uint_as_float(byte[i] << 23);
#pragma unroll
        for (int h = 0; h < LB / 4; ++h) lds_put(lds_base((in_row ^ x ^ h * 16) + at) + off, __builtin_bit_cast(u32x4, fp4x8_to_bf16(raw[i][h], f)));
      } else {
        const float f = __uint_as_float(byte[i] << 23);
#pragma unroll
        for (int h = 0; h < LB / 8; ++h)
          lds_put(lds_base((in_row ^ x ^ h * 16) + at) + off, __builtin_bit_cast(u32x4, fp8x8_to_bf16(make_uint2(raw[i][2 * h], raw[i][2 * h + 1]), f)));
      }
    }
  }
};

// A lane's place in a tile's rows for either operand, before the exchange of chunks: what selects channels is exclusive-or'ed in.
template <int HD> __device__ __forceinline__ uint32_t k_lane(int lane) { return (lane & 15) * HD * 2 + ((lane >> 4) ^ k_swizzle<HD>(lane & 15)) * 16; }
template <int HD> __device__ __forceinline__ uint32_t v_lane(int lane) {
  const int r = (lane >> 4) * 4 + ((lane >> 2) & 3);         // each group of 16 lanes hands the read four rows' 32 bytes and gets a channel a lane
  return r * HD * 2 + (((lane >> 1) & 1) ^ v_swizzle<HD>(r)) * 16 + (lane & 1) * 8;
}
// keys kt * 16 .., channels ks * 32 .. of a tile: A operand of S^T
template <int HD> __device__ __forceinline__ bf16x8 read_k(uint32_t tile, uint32_t klane, int kt, int ks) {
  return lds_get(lds_base((klane ^ (ks * 64)) + tile) + kt * 16 * HD * 2);
}
// keys s * 32 .., channels d * 16 .. of a tile: A operand of O^T.  Element e of a lane is key s * 32 + (e >> 2) * 16 + (lane >> 4) * 4 + (e & 3), as in the
// accumulators of two tiles of 16 keys.
template <int HD> __device__ __forceinline__ bf16x8 read_v(uint32_t tile, uint32_t vlane, int s, int d) {
  const uint32_t at = lds_base((vlane ^ (d * 32)) + tile) + s * 32 * HD * 2;
  return __builtin_shufflevector(lds_get_transposed(at), lds_get_transposed(at + 16 * HD * 2), 0, 1, 2, 3, 4, 5, 6, 7);
}

// Weights of KT tiles of 16 keys of a row, from scores in sc, packed for the second product.  They are rounded to bf16 (half a step: 2^-8), the type of the values
// that they meet, which the fast matrix instructions ask for; l grows by the rounded weights, so that what all have in common cancels (2.1e-3 from 64 bits at
// 9360 keys, the result's own rounding included; 1.7e-3 with fp32 weights).  The reference is m (finite, or 0 while there is none).
template <int KT> __device__ __forceinline__ void weigh(const f32x4 (&sc)[KT], float scale, float ref, float& l, uint4 (&pf)[KT / 2]) {
#pragma unroll
  for (int s = 0; s < KT / 2; ++s) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4& v = sc[2 * s + (i >> 1)];
      w[i] = pack_bf16x2(__builtin_amdgcn_exp2f(fmaf(v[2 * (i & 1)], scale, -ref)), __builtin_amdgcn_exp2f(fmaf(v[2 * (i & 1) + 1], scale, -ref)));
      l = add_pk(w[i], l);
    }
    pf[s] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// bf16 pairs: where the exponent is all ones (infinity or NaN)
__device__ __forceinline__ bool not_finite(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }
// O^T += V^T P^T of 32 keys, NT tiles of 16 rows, where a value that is not finite must not meet the weight 0 of a row that does not see its key (0 *
// infinity is NaN).  Values are multiplied with what is not finite set to 0; rows that do see +inf, -inf or NaN in a channel are found by
// products of ones and get it added.  seen: B operand of ones where the row sees the key.  Returns whether there was any such value, seen or not.
template <int HD, int NT>
__device__ __forceinline__ bool weighted_sum_checked(uint32_t tile, uint32_t vlane, int s, const uint4 (&pf)[NT], const uint4 (&seen)[NT], f32x4 (&o)[HD / 16][NT]) {
  bool met = false;
#pragma unroll
  for (int d = 0; d < HD / 16; ++d) {
    const uint4 v = __builtin_bit_cast(uint4, read_v<HD>(tile, vlane, s, d));
    const bool bad = not_finite(v.x) || not_finite(v.y) || not_finite(v.z) || not_finite(v.w);
    if (!__any(bad)) {
#pragma unroll
      for (int t = 0; t < NT; ++t) o[d][t] = mfma(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, pf[t]), o[d][t]);
      continue;
    }
    met = true;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    // one kind of value after the other: all at once would take registers from the loop around
    auto operand = [&](auto&& of) __attribute__((always_inline)) {
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = of(w[i] & 0xffffu) | of(w[i] >> 16) << 16;
      __builtin_amdgcn_sched_barrier(0);
      return __builtin_bit_cast(bf16x8, make_uint4(x[0], x[1], x[2], x[3]));
    };
    const bf16x8 finite = operand([](uint32_t x) __attribute__((always_inline)) { return (x & 0x7f80u) == 0x7f80u ? 0u : x; });
#pragma unroll
    for (int t = 0; t < NT; ++t) o[d][t] = mfma(finite, __builtin_bit_cast(bf16x8, pf[t]), o[d][t]);
    auto add = [&](auto&& of, auto&& to) __attribute__((always_inline)) {   // to(value) for rows that see one of the kind that has ones in of(bits)
      const bf16x8 kind = operand(of);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const f32x4 n = mfma(kind, __builtin_bit_cast(bf16x8, seen[t]), f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int r = 0; r < 4; ++r) o[d][t][r] = n[r] > 0.f ? to(o[d][t][r]) : o[d][t][r];
      }
    };
    add([](uint32_t x) __attribute__((always_inline)) { return x == 0x7f80u ? 0x3f80u : 0u; }, [](float y) __attribute__((always_inline)) { return y + INFINITY; });
    add([](uint32_t x) __attribute__((always_inline)) { return x == 0xff80u ? 0x3f80u : 0u; }, [](float y) __attribute__((always_inline)) { return y - INFINITY; });
    add([](uint32_t x) __attribute__((always_inline)) { return (x & 0x7fffu) > 0x7f80u ? 0x3f80u : 0u; }, [](float) __attribute__((always_inline)) { return __uint_as_float(0x7fc00000u); });
  }
  return met;
}
// ones where a score is above -inf
__device__ __forceinline__ uint4 ones_of(const f32x4& x, const f32x4& y) {
  auto pair = [](float p, float q) __attribute__((always_inline)) { return (p == -INFINITY ? 0u : 0x3f80u) | (q == -INFINITY ? 0u : 0x3f800000u); };
  return make_uint4(pair(x[0], x[1]), pair(x[2], x[3]), pair(y[0], y[1]), pair(y[2], y[3]));
}
// The rest of a tile of KT * 16 keys whose scores are in sc: what a row does not see (border), the classical online softmax (of_row: whether this tile may raise
// a row's reference), the weighted sum (checked: with values looked at; KEEP: sums that are not finite are kept).  Returns whether a value looked at was not finite.
template <int HD, int KT, int NT, bool KEEP>
__device__ __forceinline__ bool sum_tile(const PagedArgs& a, const Block& b, uint32_t vtile, f32x4 (&sc)[NT][KT], int key0, bool border, bool checked, const bool (&of_row)[NT], const int (&end)[NT], bool gaps,
                                         Soft (&z)[NT], f32x4 (&o)[HD / 16][NT], int lane) {
  uint4 pf[NT][KT / 2];
  bool met = false;
  const uint32_t gone = gaps ? missing<KT>(a, b, key0, lane) : 0;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (border) hide<KT>(sc[t], key0, end[t], gone, lane);
    float ref;
    const float alpha = raise(z[t], of_row[t] ? maximum<KT>(sc[t], KT) * a.scale : -INFINITY, ref);
    if (KEEP && __any(alpha == 0.f)) {
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) o[d][t] = lowered(o[d][t], alpha);
    } else if (!__all(alpha == 1.f)) {                       // most tiles raise no row's reference
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) o[d][t] *= alpha;
    }
    weigh<KT>(sc[t], a.scale, ref, z[t].l, pf[t]);
  }
#pragma unroll
  for (int s = 0; s < KT / 2; ++s) {
    uint4 p[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) p[t] = pf[t][s];
    if (checked) {
      uint4 seen[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) seen[t] = ones_of(sc[t][2 * s], sc[t][2 * s + 1]);
      met |= weighted_sum_checked<HD, NT>(vtile, v_lane<HD>(lane), s, p, seen, o);
    } else {
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) {
        if (NT > 1 && d % 4 == 0) __builtin_amdgcn_sched_barrier(0);         // else all values are read at once, into registers that are not there
        const bf16x8 vf = read_v<HD>(vtile, v_lane<HD>(lane), s, d);
#pragma unroll
        for (int t = 0; t < NT; ++t) o[d][t] = mfma(vf, __builtin_bit_cast(bf16x8, p[t]), o[d][t]);
      }
    }
  }
  return met;
}
// scores of a tile in plain order
template <int HD, int KT, int NT>
__device__ __forceinline__ void score_tile(uint32_t ktile, const bf16x8 (&qf)[NT][HD / 32], f32x4 (&sc)[NT][KT], int lane) {
  // one column of rows leaves registers for all operands, which are on their way before the first product; else a step's are
  constexpr int KS = HD / 32, AT_ONCE = NT == 1 ? KS : 1;
  bf16x8 kf[KS][KT];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    if (ks % AT_ONCE == 0) {
#pragma unroll
      for (int i = ks; i < ks + AT_ONCE; ++i)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) kf[i][kt] = read_k<HD>(ktile, k_lane<HD>(lane), kt, i);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int t = 0; t < NT; ++t) sc[t][kt] = mfma(kf[ks][kt], qf[t][ks], ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sc[t][kt]);
  }
}

// Codes of 4 bits of 32 keys straight from the pages into operands: a lane takes a quarter of a key's row, whole groups or half of one, as it lies there, and the
// channels of its quarter in the products' order, 8 in each: which channels meet in a product is free, as long as the queries' are the same ones (SPREAD).
template <int HD> struct KeyCodes {
  static constexpr int ROW = HD / 2;         // bytes of a row in the pages
  typedef typename std::conditional<HD == 128, u32x4, u32x2>::type Raw;
  Raw raw[2];
  uint32_t byte[2];
  __device__ __forceinline__ void load(const PagedArgs& a, const int64_t (&at)[2], int lane) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      raw[kt] = *(const Raw*)((const char*)a.data + at[kt] * ROW + (lane & 15) * ROW + (lane >> 4) * (ROW / 4));
      byte[kt] = (a.scales + at[kt] * (HD / FP4_GROUP))[(lane & 15) * (HD / FP4_GROUP) + (lane >> 4) * (HD / 4) / FP4_GROUP];
    }
  }
  template <int NT> __device__ __forceinline__ void score(const bf16x8 (&qf)[NT][HD / 32], f32x4 (&sc)[NT][2]) const {
#pragma unroll
    for (int ks = 0; ks < HD / 32; ++ks)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const bf16x8 k = __builtin_bit_cast(bf16x8, fp4x8_to_bf16(raw[kt][ks], __uint_as_float(byte[kt] << 23)));
#pragma unroll
        for (int t = 0; t < NT; ++t) sc[t][kt] = mfma(k, qf[t][ks], ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sc[t][kt]);
      }
  }
};

// SPREAD: lane group g has channels g * (HD / 4) .., as KeyCodes
template <int HD, int NT, bool SPREAD = false>
__device__ __forceinline__ void load_queries(const PagedArgs& a, const Block& b, int row0, bf16x8 (&qf)[NT][HD / 32], int (&end)[NT], int lane) {
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = row0 + t * 16 + (lane & 15);
    const bf16_t* const q = (const bf16_t*)a.q + row_at(a, b, row < b.rows ? row : b.rows - 1, a.q_ts, a.q_hs) + (lane >> 4) * (SPREAD ? HD / 4 : 8);
#pragma unroll
    for (int ks = 0; ks < HD / 32; ++ks) qf[t][ks] = __builtin_bit_cast(bf16x8, *(const uint4*)(q + ks * (SPREAD ? 8 : 32)));
    end[t] = row_end(a, b, row);
  }
}

// Few rows: NT * 16 of them, W wavefronts that deal the block's keys out in tiles of 32 (wavefront w: tiles w, w + W, ...), each through its own piece of
// LDS, the next tile on its way in registers; nobody waits for anybody until the results are joined in LDS, in wavefront order.  W = 4: two blocks to a
// CU keep 128 KB (codes: 64 KB) under way, and what bounds it is memory: 64 sequences of 16 .. 16000 keys, 8 heads of 128 in 8 bits, 201 us, 5.3 TB/s.  W = 8: no more
// blocks than CUs, bound by a trip's chain of steps, 1.6 us for 256 keys: one token over 517 keys with 12 heads 10.3 us.
// Codes of 4 bits take so little memory that two blocks on a CU are bound by their own work: keys go from the pages straight into operands (KeyCodes), which frees
// half of the LDS, and three blocks fit, four with heads of 64: the same 64 sequences, 32 heads on 8, 156 us, 143 with keys straight into operands, 127 with three blocks (4.9 TB/s beside
// plan and join).  32 rows of heads of 64 leave registers for three: 64 sequences of 16000 keys, 128 heads on 4, 100 -> 91 us; of heads of 128 for two, three spill 400 bytes a lane.
constexpr int few_per_cu(int head_dim, int nt, int format) { return format != DP_KV_FP4 ? 2 : head_dim == 64 && nt == 1 ? 4 : head_dim == 64 || nt == 1 ? 3 : 2; }
template <int HD, int NT, int W, int FORMAT, bool PLAN>
__global__ __launch_bounds__(W * 64, (W == 4 ? few_per_cu(HD, NT, FORMAT) : 2)) void k_paged_few(const PagedArgs a) {
  constexpr int QB = NT * 16, KT = 2, CR = HD / 8, TILE = 32 * CR, JOIN = (W * 16 * (2 + HD + 4) * 4 + 15) / 16;
  constexpr bool DIRECT = FORMAT == DP_KV_FP4;               // keys do not go through LDS
  constexpr int TILES = W * (DIRECT ? 1 : 2) * TILE;
  __shared__ uint4 smem[TILES > JOIN ? TILES : JOIN];
  static_assert(sizeof(smem) >= sizeof(float) * W * 16 * (2 + HD + 4), "join_waves");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t kt = lds_address(smem) + wave * (DIRECT ? 1 : 2) * TILE * 16, vt = DIRECT ? kt : kt + TILE * 16;
  const int64_t to_values = (int64_t)a.hk << a.page_shift;
  Walk<QB, 128, PLAN> walk(a, blockIdx.x);
  Piece p;
  if (!walk.next(a, p)) return;
  do {
    if constexpr (PLAN) __syncthreads();                     // the piece before is done with LDS
    const int lane = fresh_lane();
    const Block& b = p.b;
    bf16x8 qf[NT][HD / 32];
    int end[NT];
    load_queries<HD, NT, DIRECT>(a, b, b.first, qf, end, lane);
    Soft z[NT];
    f32x4 o[HD / 16][NT];
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        z[t] = Soft{-INFINITY, 0.f};
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) o[d][t] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    };
    clear();
    typedef Carry<HD, 32, 1, FORMAT> Tile;
    typename std::conditional<DIRECT, KeyCodes<HD>, Tile>::type ck;
    Tile cv;
    int key = p.k0 + wave * 32;
    auto load = [&](int at, int lane) __attribute__((always_inline)) {
      const auto rows = Tile::rows(a, b, at, 0);
      if constexpr (DIRECT) {
        static_assert(sizeof(rows.at) == 16, "two groups of 16 keys");
        ck.load(a, rows.at, lane);
      } else {
        ck.load(a, rows, 0, 0, lane);
      }
      cv.load(a, rows, to_values, 0, lane);
    };
    if (key < p.k1) load(key, lane);
    const bool gaps = __builtin_amdgcn_readfirstlane((int)pages_missing(a, b, p.k0, p.k1));
    // the tile in the registers; `next` sends the one after it on its way
    auto tile = [&](auto careful, int lane, auto&& next) __attribute__((always_inline)) {
      f32x4 sc[NT][KT];
      if constexpr (DIRECT) {
        ck.score(qf, sc);
        cv.template store<true>(vt, 0, lane);
        next();
      } else {
        ck.template store<false>(kt, 0, lane);
        cv.template store<true>(vt, 0, lane);
        next();
        score_tile<HD, KT, NT>(kt, qf, sc, lane);
      }
      bool all[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) all[t] = true;
      const bool border = key + 32 > b.whole || gaps;
      sum_tile<HD, KT, NT, careful>(a, b, vt, sc, key, border, border || careful, all, end, gaps, z, o, lane);
    };
    for (; key < p.k1; key += W * 32) tile(std::false_type{}, lane, [&]() __attribute__((always_inline)) { if (key + W * 32 < p.k1) load(key + W * 32, lane); });
    if (!__all(finite(o))) {
      clear();
      for (key = p.k0 + wave * 32; key < p.k1; key += W * 32) {
        const int lane = fresh_lane();
        load(key, lane);
        tile(std::true_type{}, lane, []() {});
      }
    }
    join_waves<bf16_t, HD, NT, W, false>(a, b, (float*)smem, z, o, p.slot, wave, lane);
  } while (PLAN && walk.next(a, p));
}

// LDS by typed address.  In the loop over whole tiles, tiles arrive by direct loads while others are read; what says that the two do not meet are the
// restricted pointers of `round`, without which the compiler has every read of LDS wait for all loads on their way.
typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ bf16x8 lds_get(const lds_char* p) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_bit_cast(bf16x8, *(const __attribute__((address_space(3))) u32x4*)p);
#else
  return bf16x8{};
#endif
}
__device__ __forceinline__ bf16x8 lds_get_v(const lds_char* p, int u_bytes) {
#ifdef __HIP_DEVICE_COMPILE__
  const bf16x4 a = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p));
  const bf16x4 b = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p + u_bytes)));
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
#else
  return bf16x8{};
#endif
}
// this wavefront's LDS traffic is done, and none of what is written before the barrier moves behind it or the other way round
__device__ __forceinline__ void turn() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// A tile of 64 keys or values on its way from the pages into LDS by direct loads: 64 lanes of 16 bytes a trip, whose places in the rows are
// exchanged at the source.
template <int HD, int W> struct Direct {
  static constexpr int CR = HD / 8, RW = 64 / CR, N = HD / (W * 8);          // chunks and rows of a trip of one wavefront, trips
  static_assert(N * W * RW == 64 && (W * RW) % 16 == 0, "the same exchange in every trip");
  uint32_t k, v;                             // this lane's place in a trip's rows
  __device__ __forceinline__ Direct(int w, int lane) {
    const int row = w * RW + lane / CR, c = lane % CR;
    k = (lane / CR) * HD * 2 + ((c ^ k_swizzle<HD>(row)) * 16);
    v = (lane / CR) * HD * 2 + ((c ^ v_swizzle<HD>(row)) * 16);
  }
  template <typename Rows> static __device__ __forceinline__ void load(const PagedArgs& a, const Rows& rows, int64_t to_values, uint32_t place, lds_char* tile, int w) {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const char* const from = (const char*)a.data + (rows.row(i, w) + to_values) * (HD * 2);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void*)from, 0, 0x7fffffff, 0x00020000), (lds_void_t*)(tile + (i * W + w) * 1024), 16, place, 0, 0, 0);
    }
#endif
  }
};

// What a wavefront of k_paged_turns has in registers through its whole tiles.
template <int HD> struct State {
  static constexpr int KS = HD / 32, DT = HD / 16;
  bf16x8 qf[2][KS], kf[2][4], vf[2][4];      // operands two steps of the head dim, two groups of four values' tiles ahead
  f32x4 o[DT][2], sc[2][4];
  uint4 pf[2][2];
  Soft z[2];
  float ref[2];
  uint32_t klane, vlane;
  // keys at channels ks * 32 ..; the g-th four of the values' tiles (32-key half f / DT, channels f % DT * 16 ..)
  template <int ks> __device__ __forceinline__ void read_keys(const lds_char* tile) {
    const lds_char* const p = tile + (klane ^ (ks * 64));
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) kf[ks & 1][kt] = lds_get(p + kt * 16 * HD * 2);
  }
  template <int g> __device__ __forceinline__ void read_values(const lds_char* tile) {
#pragma unroll
    for (int i = 0; i < 4; ++i) vf[g & 1][i] = lds_get_v(tile + (vlane ^ ((g * 4 + i) % DT * 32)) + (g * 4 + i) / DT * 32 * HD * 2, 16 * HD * 2);
  }
  template <int ks> __device__ __forceinline__ void score_step() {
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
      for (int t = 0; t < 2; ++t) sc[t][kt] = mfma(kf[ks & 1][kt], qf[t][ks], ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sc[t][kt]);
  }
  template <int g> __device__ __forceinline__ void sum_step() {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t) o[(g * 4 + i) % DT][t] = mfma(vf[g & 1][i], __builtin_bit_cast(bf16x8, pf[t][(g * 4 + i) / DT]), o[(g * 4 + i) % DT][t]);
  }
  __device__ __forceinline__ void weights(float scale) {
#pragma unroll
    for (int t = 0; t < 2; ++t) weigh<4>(sc[t], scale, ref[t], z[t].l, pf[t]);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      z[t] = Soft{-INFINITY, 0.f};
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
};

// The turn of products: scores of the tile whose keys are at k1 (its first two steps are in kf), weighted sum of the one whose values are at v0
template <int HD> __device__ __forceinline__ void products(State<HD>& s, const lds_char* k1, const lds_char* v0) {
  constexpr int KS = HD / 32;
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("" : "+v"(s.klane), "+v"(s.vlane));   // a dozen addresses made of them each time, not kept in registers that the loop has none of
#endif
  __builtin_amdgcn_s_setprio(1);
  static_for<KS>([&](auto k_) __attribute__((always_inline)) {
    constexpr int ks = decltype(k_)::value;
    s.template score_step<ks>();
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (ks + 2 < KS) s.template read_keys<ks + 2>(k1);
    else s.template read_values<ks + 2 - KS>(v0);
    __builtin_amdgcn_sched_barrier(0);
  });
  static_for<KS>([&](auto g_) __attribute__((always_inline)) {
    constexpr int g = decltype(g_)::value;
    s.template sum_step<g>();
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (g + 2 < KS) s.template read_values<g + 2>(v0);
    __builtin_amdgcn_sched_barrier(0);
  });
  __builtin_amdgcn_s_setprio(0);
  __builtin_amdgcn_sched_barrier(0);
}
// Round j of the loop over whole tiles: the turn of exponentials (weights of tile j + 1, the first keys of tile j + 2), in which `move` sends tiles to come on
// their way to k_to and v_to; then the turn of products (scores of tile j + 2, weighted sum of tile j + 1).
template <int HD, typename Move, typename Between>
__device__ __forceinline__ void round(State<HD>& s, float scale, const lds_char* __restrict__ k2, const lds_char* __restrict__ v1, lds_char* __restrict__ k_to,
                                      lds_char* __restrict__ v_to, Move&& move, Between&& between) {
  s.template read_keys<0>(k2);
  s.template read_keys<1>(k2);
  __builtin_amdgcn_sched_barrier(0);
  move(k_to, v_to);
  __builtin_amdgcn_sched_barrier(0);
  s.weights(scale);
  __builtin_amdgcn_sched_barrier(0);
  between();
  products(s, k2, v1);
}

// Many rows: wavefronts of 32 rows (two columns of 16) that share key tiles of 64.  WIDE: eight of them, 256 rows, one block to a CU, whose halves (0-3 and
// 4-7) are half a round apart, with a barrier at every turn: of the two wavefronts of a SIMD one multiplies while the other does exponentials.
// Else four, 128 rows, two blocks to a CU, which do the same for each other as it comes, one barrier a round; what a block does before and after its
// tiles hides behind the other.
// Rows as they are come by direct loads into LDS (four stages, or two); codes through registers, converted on the way (three, or two).
// The softmax's reference is fixed to a row's maximum over the first 32 keys: weights (bf16) and fp32 sums have 8 exponent bits, so nothing is lost until
// a sum, of weights or of weighted values, is beyond 2^100; a block with such a row, or one that is not finite, is done again tile by tile, with the reference of those rows raised as in the
// classical online softmax (the other rows get the same bits).  So are the tiles that hold a border, for all rows.
// What bounds it: the matrix pipes, where blocks fill the chip.  6240 x 9360 x 40 heads of 128 in 8 bits 1010 us, 1.18 PFLOP/s; 1560 x 20280 x 12 as they are in
// three ranges 194 us, 9 of them joining, 1.0; heads of 64, 8192 x 8192 x 32, 519 us, 1.06.
template <int HD, bool WIDE, int FORMAT>
__global__ __launch_bounds__(WIDE ? 512 : 256, 2) void k_paged_turns(const PagedArgs a) {
  constexpr bool CODES = FORMAT != DP_KV_PLAIN;
  constexpr int KS = HD / 32, DT = HD / 16, TILE = 64 * HD * 2;   // bytes
  constexpr int W = WIDE ? 8 : 4, QB = W * 32, NS = WIDE ? (CODES ? 3 : 4) : 2;   // wavefronts, rows of a block, LDS stages of keys and of values
  extern __shared__ uint4 smem[];            // NS key tiles, NS value tiles
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // blocks are handed out to the eight XCDs in turn: each gets a run of tiles, whose neighbours share keys in its L2, a head's first ranges before its second ones
  const int of_head = a.tiles * a.parts, total = of_head * a.hk, per = (total + 7) >> 3;
  const int pid = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3), hk = pid / of_head, part = (pid - hk * of_head) / a.tiles;
  if ((int)(blockIdx.x >> 3) >= per || pid >= total) return;
  Walk<QB, 64, false> walk(a, pid - hk * of_head - part * a.tiles + hk * a.tiles, part);
  Piece p;
  if (!walk.next(a, p)) return;
  const Block& b = p.b;
  // tiles of this range: whole ones from t0 on, then those with a border up to t1
  const int t0 = p.k0 / 64, t1 = (p.k1 + 63) / 64;
  int whole = (b.whole < p.k1 ? b.whole : p.k1) / 64 - t0;
  if (whole < 0) whole = 0;
  bool gaps = false;
  const uint32_t kst = lds_address(smem), vst = kst + NS * TILE;
  lds_char* const kst_ = (lds_char*)(lds_void_t*)smem;
  lds_char* const vst_ = kst_ + NS * TILE;
  const int64_t to_values = (int64_t)a.hk << a.page_shift;
  typedef Carry<HD, 64, W, FORMAT> Registers;
  Registers ck, cv;
  typedef Direct<HD, W> Loads;
  const Loads direct(wave, lane);
  // tiles past the range: its first again, never used
  auto rows_of = [&](int j) __attribute__((always_inline)) { return Registers::rows(a, b, (t0 + j < t1 ? t0 + j : t0) * 64, wave); };
  typedef decltype(rows_of(0)) Rows;
  auto direct_k = [&](const Rows& rows, lds_char* to) __attribute__((always_inline)) { Loads::load(a, rows, 0, direct.k, to, wave); };
  auto direct_v = [&](const Rows& rows, lds_char* to) __attribute__((always_inline)) { Loads::load(a, rows, to_values, direct.v, to, wave); };
  auto load_k = [&](const Rows& rows) __attribute__((always_inline)) { ck.load(a, rows, 0, wave, lane); };
  auto load_v = [&](const Rows& rows) __attribute__((always_inline)) { cv.load(a, rows, to_values, wave, lane); };
  auto store_k = [&](int j) __attribute__((always_inline)) { ck.template store<false>(kst + (j % NS) * TILE, wave, lane); };
  auto store_v = [&](int j) __attribute__((always_inline)) { cv.template store<true>(vst + (j % NS) * TILE, wave, lane); };
  auto load_both = [&](int at) __attribute__((always_inline)) {
    const Rows both = Registers::rows(a, b, at * 64, wave);
    load_k(both); load_v(both);
  };
  auto kt = [&](int j) __attribute__((always_inline)) { return kst_ + (j % NS) * TILE; };
  auto vt = [&](int j) __attribute__((always_inline)) { return vst_ + (j % NS) * TILE; };

  // Round j sends keys of tile j + AHEAD and values of the one before it, whose place in the pages it has from the round before.  Direct loads land a round
  // later, or (four stages) two; from registers, tiles go into LDS a round later and into the matrix pipe two.
  constexpr int AHEAD = CODES || WIDE ? 4 : 3;
  // what the first scores need, on its way before the queries and the look at the pages
  Rows rows{};
  if (p.k0 < p.k1) rows = rows_of(0);                         // a sequence without keys has no entry in the table to look at
  bool loaded = p.k0 < p.k1 && (CODES || whole == 0);         // whether `tile`, the next that goes through registers in the end, is in them
  if (loaded) {
    load_k(rows); load_v(rows);
  } else if (whole > 0) {
#pragma unroll
    for (int j = 0; j < AHEAD - 1; ++j) {
      direct_k(rows, kt(j)); direct_v(rows, vt(j));
      rows = rows_of(j + 1);
    }
    if constexpr (WIDE) direct_k(rows, kt(3));
  }
  State<HD> s;
  int end[2];
  load_queries<HD, 2>(a, b, b.first + wave * 32, s.qf, end, lane);
  s.klane = k_lane<HD>(lane);
  s.vlane = v_lane<HD>(lane);
  if (__builtin_amdgcn_readfirstlane((int)pages_missing(a, b, p.k0, p.k1))) {
    if (!CODES && whole > 0) { vm_wait<0>(); __syncthreads(); }   // nothing lands in LDS any more
    whole = 0;
    gaps = true;
  }
  s.clear();
  int tile = t0;
  bool over[2] = {};                         // rows whose sums leave no room for their reference, or are not finite
  auto find_over = [&](auto&& is) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      int bad = is(over_lanes(s.z[t].l));
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) bad |= is(s.o[d][t][r]);
      bad |= __shfl_xor(bad, 16, 64);
      over[t] = bad | __shfl_xor(bad, 32, 64);
    }
  };
  bool scored = false;                       // whether the scores of `tile` are there, and its values in LDS
  if (whole > 0) {
    if constexpr (CODES) {
      rows = rows_of(1);
      store_k(0); store_v(0);
      load_k(rows); load_v(rows);
      rows = rows_of(2);
      store_k(1); store_v(1);
      load_k(rows); load_v(rows);
      rows = rows_of(3);
    } else {
      vm_wait<0>();
    }
    turn();
    static_for<KS>([&](auto k_) __attribute__((always_inline)) {
      constexpr int ks = decltype(k_)::value;
      s.template read_keys<ks>(kt(0));
      s.template score_step<ks>();
    });
#pragma unroll
    for (int t = 0; t < 2; ++t) s.z[t].m = s.ref[t] = maximum<4>(s.sc[t], 2) * a.scale;
    s.weights(a.scale);
    s.template read_keys<0>(kt(1));
    s.template read_keys<1>(kt(1));
    turn();
    if constexpr (CODES) {
      store_k(2);
      load_k(rows);
    } else if constexpr (!WIDE) {
      direct_k(rows, kt(2));
    }
    if (WIDE && wave >= 4) turn();           // the second half starts half a round later
    products(s, kt(1), vt(0));
    if constexpr (!CODES && !WIDE) vm_wait<0>();
    turn();
    for (int j = 0; j < whole - 1; ++j) {
      const Rows before = rows;              // the pages' table is read before the rows are asked for
      rows = rows_of(j + AHEAD);
      round(s, a.scale, kt(j + 2), vt(j + 1), kt(j + AHEAD), vt(j + AHEAD - 1),
            [&](lds_char* k_to, lds_char* v_to) __attribute__((always_inline)) {
              if constexpr (CODES) {
                store_k(j + 3);
                store_v(j + 2);
                __builtin_amdgcn_sched_barrier(0);
                load_v(before);
                load_k(rows);
              } else {
                direct_v(before, v_to);
                direct_k(rows, k_to);
              }
            },
            [&]() __attribute__((always_inline)) {
              if constexpr (!CODES && WIDE) vm_wait<2 * Loads::N>();   // what was requested a round ago
              if constexpr (WIDE) turn();
            });
      if constexpr (!CODES && !WIDE) vm_wait<0>();            // what was requested in this round
      turn();
    }
    if constexpr (!CODES) vm_wait<0>();      // nothing lands in LDS any more
    // of the first tile with a border, the scores are there and the values in LDS; the one after it goes on its way
    tile = t0 + whole;
    loaded = tile + 1 < t1;
    if (loaded) load_both(tile + 1);
    if (WIDE && wave < 4) turn();            // the halves meet again
    find_over([&](float x) __attribute__((always_inline)) { return !(fabsf(x) <= 0x1p100f); });
    scored = !__syncthreads_or(over[0] || over[1]);
  }
  // tile by tile, the next one on its way, in stages 0 and 1 in turn: what is left, or with `careful` everything once more
  bool met = false;                          // whether a value in a tile with a border is not finite: all wavefronts go through the same tiles
  auto tiles = [&](auto careful) __attribute__((always_inline)) {
    for (int j = 0; tile < t1; ++j, ++tile) {
      uint32_t values = vst + (whole % NS) * TILE;
      if (!scored) {
        if (!loaded) load_both(tile);
        store_k(j & 1); store_v(j & 1);
        loaded = tile + 1 < t1;
        if (loaded) load_both(tile + 1);
        __syncthreads();
        score_tile<HD, 4, 2>(kst + (j & 1) * TILE, s.qf, s.sc, lane);
        values = vst + (j & 1) * TILE;
      }
      const bool border = tile >= t0 + whole, of_row[2] = {!careful || border || over[0], !careful || border || over[1]};
      met |= sum_tile<HD, 4, 2, careful>(a, b, values, s.sc, tile * 64, !careful || border, true, of_row, end, gaps, s.z, s.o, lane);
      if (scored) { scored = false; __syncthreads(); }        // stages are written again
    }
  };
  bool once_more = whole > 0 && !scored;
  if (!once_more) {
    tiles(std::false_type{});
    if (met) {
      find_over([&](float x) __attribute__((always_inline)) { return !(fabsf(x) < INFINITY); });
      once_more = __syncthreads_or(over[0] || over[1]);
    }
  }
  if (__builtin_expect(once_more, 0)) {
    s.clear();
#pragma unroll
    for (int t = 0; t < 2; ++t) s.z[t].m = over[t] || whole == 0 ? -INFINITY : s.ref[t];
    tile = t0;
    loaded = false;
    tiles(std::true_type{});
  }
  const float l[2] = {over_lanes(s.z[0].l), over_lanes(s.z[1].l)};
  if (p.slot >= 0) {
    float* const ps = a.partial + (size_t)p.slot * (QB * (2 + HD));
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int row = wave * 32 + t * 16 + lr;
      if (b.first + row >= b.rows) continue;
      if (lg == 0) { ps[row] = s.z[t].m; ps[QB + row] = l[t]; }
      put_row<HD, 2, false>(ps + 2 * QB + row * HD, s.o, t, lg, 1.f);
    }
  } else {
    // a lane holds 4 consecutive channels of a row per accumulator tile.  The 32 x HD tile of this wavefront goes through LDS (a wavefront
    // only touches its own rows, and LDS serves a wavefront's accesses in order) so that global memory sees whole rows, 16 bytes
    // per lane.  8-byte units are exchanged by the row.
    constexpr int UPR = HD / 4, CPR = HD / 8, RPI = 64 / CPR;      // units, 16-byte chunks per row; rows per read
    __syncthreads();
    uint2* const stg = (uint2*)smem + wave * 32 * UPR;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float inv = inverse(l[t]);
      const int row = t * 16 + lr;
#pragma unroll
      for (int d = 0; d < DT; ++d)
        stg[row * UPR + ((d * 4 + lg) ^ (row & (UPR - 1)))] = make_uint2(pack_bf16x2(s.o[d][t][0] * inv, s.o[d][t][1] * inv), pack_bf16x2(s.o[d][t][2] * inv, s.o[d][t][3] * inv));
    }
    const uint4* const stg16 = (const uint4*)stg;
#pragma unroll
    for (int it = 0; it < 32 / RPI; ++it) {
      const int row = it * RPI + lane / CPR, ch = lane % CPR;
      uint4 dv = stg16[row * CPR + ch];
      // units 2 ch and 2 ch + 1 of the exchanged row are the halves of chunk ch ^ (exchange >> 1), the other way round for odd rows
      if (row & 1) dv = make_uint4(dv.z, dv.w, dv.x, dv.y);
      const int c = ch ^ ((row & (UPR - 1)) >> 1), r = b.first + wave * 32 + row;
      if (r < b.rows) *(uint4*)((bf16_t*)a.out + row_at(a, b, r, a.o_ts, a.o_hs) + c * 8) = dv;
    }
  }
}

Route route(const PagedArgs& a, int head_dim, int format) {
  Route r{};
  const int64_t rows = (int64_t)a.max_q * a.shared, keys = a.max_kv;          // of a sequence, at most
  r.parts = 1;
  r.part_keys = (int)keys;
  if (rows <= 32) {
    r.qb = rows <= 16 ? 16 : 32;
    r.tiles = tiles_of_call(a, r.qb);
    const int64_t units = (keys + 127) / 128, blocks = r.tiles * a.hk;
    if (a.n_seqs == 1 || units <= 16 || blocks * keys <= 400000) {
      // Ranges for one block of eight wavefronts a CU, no shorter than one of their trips (256 keys), from three on: one token of 12 heads of 128 over 767 keys 11.5 us
      // in one, over 768 10.2 in three.
      int64_t parts = (keys + 255) / 256;
      if (parts > 256 / blocks) parts = 256 / blocks;
      if (keys >= 768 && parts > 1) {
        r.part_keys = (int)(((keys + parts - 1) / parts + 31) / 32 * 32);
        r.parts = (int)((keys + r.part_keys - 1) / r.part_keys);
      }
    } else if (blocks < 8192 && blocks * units < INT_MAX) {
      // Equal runs of all sequences' keys, as many blocks as a CU holds (few_per_cu), where there is so much work that lengths below the bound count for more than a plan: 64 sequences of 100 to
      // 16000 keys 215 us.  Equal lengths lose little: 8 of 16000 keys with 8 heads 51 us, in ranges 47; 4 of 6000 23 and 17.  Not for sequences up to 2048
      // keys (64 of 2000 52 and 44), nor for very many; units are counted in 32 bits.
      const int64_t most = 256 * few_per_cu(head_dim, rows <= 16 ? 1 : 2, format);
      r.runs = (int)(blocks * units < most ? blocks * units : most);
    }
  } else {
    // Measured, heads of 128, with 256 and 128 rows: 6240 x 9360 x 40 as they are 997 and 1032 us, in 8 bits 1027 and 1085; 1560 x 20280 x 12 in ranges 199 and 197; 1000,
    // 3000 and 2000 new tokens over up to 2000 older ones, 16 heads, causal, 214 and 197.  Heads of 64 have 128 rows at every size: two such blocks on a CU take less
    // a step than one of 256 rows (8192 x 8192 x 32: 532 us, 553).
    static const Kind wide[2] = {{256, 64, 8, 1, 1, {157}, 800}, {128, 64, 8, 2, 1, {130, 163}, 600}}, narrow{128, 64, 8, 2, 1, {80, 94}, 600};
    if (head_dim == 128) choose(a, wide, 2, head_dim, r);
    else choose(a, &narrow, 1, head_dim, r);
  }
  r.tiles_of_seq = (rows + r.qb - 1) / r.qb;
  return r;
}

template <int HD, int NT, int FORMAT> void few(const PagedArgs& a, hipStream_t st) {
  constexpr int QB = NT * 16;
  const int64_t blocks = (int64_t)a.tiles * a.hk * a.parts;
  if (a.plan) {
    k_paged_plan<QB, 128><<<1, 1024, 0, st>>>(a);
    k_paged_few<HD, NT, 4, FORMAT, true><<<(unsigned)a.runs, 256, 0, st>>>(a);
  } else if (blocks <= 256 && a.max_kv > 128) {
    k_paged_few<HD, NT, 8, FORMAT, false><<<(unsigned)blocks, 512, 0, st>>>(a);
  } else {
    k_paged_few<HD, NT, 4, FORMAT, false><<<(unsigned)blocks, 256, 0, st>>>(a);
  }
}
template <int HD, bool WIDE, int FORMAT> void turns(const PagedArgs& a, hipStream_t st) {
  constexpr int lds = (WIDE ? (FORMAT != DP_KV_PLAIN ? 3 : 4) : 2) * 2 * 64 * HD * 2;
  static std::atomic<uint64_t> done;
  allow_dynamic_lds((const void*)k_paged_turns<HD, WIDE, FORMAT>, lds, done);
  const int64_t total = (int64_t)a.tiles * a.hk * a.parts;
  k_paged_turns<HD, WIDE, FORMAT><<<(unsigned)((total + 7) / 8 * 8), WIDE ? 512 : 256, lds, st>>>(a);
}
template <int HD, int FORMAT> void launch(const PagedArgs& a, int qb, hipStream_t st) {
  if (qb == 16) { few<HD, 1, FORMAT>(a, st); launch_join<bf16_t, HD, 16>(a, st); }
  else if (qb == 32) { few<HD, 2, FORMAT>(a, st); launch_join<bf16_t, HD, 32>(a, st); }
  else if (qb == 128) { turns<HD, false, FORMAT>(a, st); launch_join<bf16_t, HD, 128>(a, st); }
  else if constexpr (HD == 128) { turns<HD, true, FORMAT>(a, st); launch_join<bf16_t, HD, 256>(a, st); }
}

}  // namespace

Route route_attn_paged_bf16(const PagedArgs& a, int head_dim, int format) { return route(a, head_dim, format); }
void launch_attn_paged_bf16(const PagedArgs& a, const Route& r, int head_dim, int format, hipStream_t st) {
  auto of = [&](auto f) {
    if (head_dim == 128) launch<128, decltype(f)::value>(a, r.qb, st); else launch<64, decltype(f)::value>(a, r.qb, st);
  };
  if (format == DP_KV_FP4) of(std::integral_constant<int, DP_KV_FP4>{});
  else if (format == DP_KV_FP8) of(std::integral_constant<int, DP_KV_FP8>{});
  else of(std::integral_constant<int, DP_KV_PLAIN>{});
}
