// What the attention kernels over a paged cache share: a call's arguments, which rows and keys a block of them owns, the way from a key
// to its row in the pages.
#pragma once
#include <limits.h>

#include "paged.h"

struct PagedArgs {
  const void* data;
  const uint8_t* scales;
  const void* q;
  void* out;
  int64_t q_ts, q_hs, o_ts, o_hs, n_tokens;
  const int32_t *q_start, *kv_len, *table;
  int32_t n_pages, page_shift, hk, shared, n_seqs, max_q, max_kv, table_width, group;
  float scale;                            // of the scores, times log2(e): softmax in powers of two
  // The launch: tiles of rows (of all sequences) and the most a sequence has.  A block has one tile's range of keys with one key head: of `parts` ranges
  // of part_keys keys each.  Or, with a plan (sequences of one tile each), the work of all tiles and heads lies in one line, in units of a number of keys, and
  // each of `runs` blocks has an equal run of it: the end of one tile's keys, all of some, the beginning of another's.
  int32_t tiles, tiles_of_seq, parts, part_keys, runs;
  int32_t* plan;                          // null, or units before each tile and of all [tiles + 1]
  float* partial;                         // of each range, or of the incomplete first [0] and last [1] tile of each run: m[QB], l[QB], O[QB][head_dim]
};

// read through the scalar cache: uniform addresses of arrays that this launch does not write (the plan is an earlier launch's)
__device__ __forceinline__ int32_t uniform_i32(const int32_t* p) {
#ifdef __HIP_DEVICE_COMPILE__
  return *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)p;
#else
  return *p;
#endif
}

// the lane, read anew for each piece of work: what is made of it is not kept in registers from one piece to the next
__device__ __forceinline__ int fresh_lane() {
  int lane = threadIdx.x & 63;
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("" : "+v"(lane));
#endif
  return lane;
}

// a sequence's new tokens and keys, whatever the arrays hold
struct Seq { int row0, n, rows, keys; };  // first row of q, new tokens, those of them within max_q, keys
__device__ __forceinline__ Seq sequence(const PagedArgs& a, int32_t q0, int32_t q1, int32_t kv) {
  const int most = (int)a.n_tokens;
  const int r0 = q0 < 0 ? 0 : q0 > most ? most : q0, r1 = q1 < r0 ? r0 : q1 > most ? most : q1;
  return Seq{r0, r1 - r0, r1 - r0 < a.max_q ? r1 - r0 : a.max_q, kv < 0 ? 0 : kv};
}
__device__ __forceinline__ Seq sequence(const PagedArgs& a, int b) {
  return sequence(a, uniform_i32(a.q_start + b), uniform_i32(a.q_start + b + 1), uniform_i32(a.kv_len + b));
}
// keys that the table holds, within the bound
__device__ __forceinline__ int held_keys(const PagedArgs& a, int keys) {
  const int64_t most = (int64_t)a.table_width << a.page_shift;
  const int k = keys < a.max_kv ? keys : a.max_kv;
  return k < most ? k : (int)most;
}
// keys that the i-th of n new tokens sees
__device__ __forceinline__ int seen_keys(const PagedArgs& a, int i, int n, int keys) {
  if (a.group == 0) return keys;
  const int p = keys - n + i;             // > -2^24
  if (p < 0) return 0;
  const int64_t end = ((int64_t)((uint32_t)p / (uint32_t)a.group) + 1) * a.group;
  return end < keys ? (int)end : keys;
}

// Rows and keys: a tile of QB rows of a sequence, with key head `hk`.  Rows are (new token, shared head) pairs.
struct Block {
  int b, hk;                              // sequence, key head
  int first, rows;                        // the tile's first row and one past the sequence's last
  Seq s;
  int held;                               // keys that exist for this sequence
  int end, whole;                         // keys that the last row sees, that the first row (and so every row) sees
};
// the rb-th tile of sequence b; false: there is none
template <int QB> __device__ __forceinline__ bool tile_of(const PagedArgs& a, Block& k, int b, int rb, int hk) {
  k.b = b;
  k.hk = hk;
  k.s = sequence(a, b);
  k.rows = k.s.rows * a.shared;
  const int of_seq = (k.rows + QB - 1) / QB;
  if (rb >= of_seq) return false;
  // the last tile of a sequence first: under a causal border it has the most keys
  k.first = (of_seq - 1 - rb) * QB;
  k.held = held_keys(a, k.s.keys);
  const int last = (k.first + QB < k.rows ? k.first + QB : k.rows) - 1;
  const int e = seen_keys(a, last / a.shared, k.s.n, k.s.keys), w = seen_keys(a, k.first / a.shared, k.s.n, k.s.keys);
  k.end = e < k.held ? e : k.held;
  k.whole = w < k.held ? w : k.held;
  return true;
}
// What is the same in all lanes goes into scalar registers, so that page tables are read through the scalar cache.
__device__ __forceinline__ void make_uniform(Block& k) {
  k.b = __builtin_amdgcn_readfirstlane(k.b);
  k.hk = __builtin_amdgcn_readfirstlane(k.hk);
  k.first = __builtin_amdgcn_readfirstlane(k.first);
  k.end = __builtin_amdgcn_readfirstlane(k.end);
  k.whole = __builtin_amdgcn_readfirstlane(k.whole);
}
// Tile `tile` of all.  false: nothing to do.  Uniform; called by whole wavefronts.
template <int QB> __device__ __forceinline__ bool locate(const PagedArgs& a, int tile, int hk, Block& k) {
  int b = -1, rb = 0;
  if (a.tiles_of_seq == 1) b = tile;
  else if (a.n_seqs == 1) { b = 0; rb = tile; }
  else {
    // tiles are numbered through the sequences: 64 of them at a time, a lane each
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
      const int sq = s0 + lane < a.n_seqs ? s0 + lane : a.n_seqs - 1;
      const Seq s = sequence(a, a.q_start[sq], a.q_start[sq + 1], 0);
      const int n = s0 + lane < a.n_seqs ? (int)(((int64_t)s.rows * a.shared + QB - 1) / QB) : 0;
      int upto = n;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) { const int v = __shfl_up(upto, o, 64); if (lane >= o) upto += v; }
      const unsigned long long beyond = __ballot(base + upto > tile);
      if (beyond) {
        const int l = __builtin_ctzll(beyond);
        b = s0 + l;
        rb = tile - base - (__shfl(upto, l, 64) - __shfl(n, l, 64));
        break;
      }
      base += __shfl(upto, 63, 64);
    }
  }
  b = __builtin_amdgcn_readfirstlane(b);
  rb = __builtin_amdgcn_readfirstlane(rb);
  hk = __builtin_amdgcn_readfirstlane(hk);
  if (b < 0 || !tile_of<QB>(a, k, b, rb, hk)) return false;
  make_uniform(k);
  return true;
}

// sums over a block of 1024 threads of what lies before each; total: of all
__device__ __forceinline__ int before(int v, int* waves, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) { const int x = __shfl_up(upto, o, 64); upto += lane >= o ? x : 0; }
  __syncthreads();
  if (lane == 63) waves[wave] = upto;
  __syncthreads();
  int base = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) { base += w < wave ? waves[w] : 0; total += waves[w]; }
  return base + upto - v;
}
// Writes the plan of a call: one block, 3 to 5 us, of them a launch and one chain of loads.  UNIT keys are a unit; a sequence that sees no key has one, a sequence without new tokens has none.
template <int QB, int UNIT>
__global__ __launch_bounds__(1024) void k_paged_plan(const PagedArgs a) {
  __shared__ int waves[16];
  int sum = 0;
  for (int t0 = 0; t0 < a.tiles; t0 += 1024) {
    const int t = t0 + (int)threadIdx.x;
    int n = 0, total;
    Block k;
    if (t < a.tiles && tile_of<QB>(a, k, t, 0, 0)) n = k.end > 0 ? (k.end + UNIT - 1) / UNIT : 1;
    const int at = sum + before(n, waves, total);
    if (t < a.tiles) a.plan[t] = at;
    sum += total;
  }
  if (threadIdx.x == 0) a.plan[a.tiles] = sum;
}

// The work of one block, piece by piece: a tile's keys [k0, k1) with a head.
struct Piece { Block b; int k0, k1, slot; };   // slot: of the partial result, or -1: these are all of the tile's keys
// `all` units, at least one, are cut into a.runs runs, or as many as there are units, none empty: run g begins at unit first_of(g); run_of(x) is the one that
// unit x lies in
__device__ __forceinline__ int64_t runs_of(const PagedArgs& a, int64_t all) { return all < a.runs ? all : a.runs; }
__device__ __forceinline__ int64_t first_of(const PagedArgs& a, int g, int64_t all) { return g * all / runs_of(a, all); }
__device__ __forceinline__ int run_of(const PagedArgs& a, int64_t x, int64_t all) { return (int)(((x + 1) * runs_of(a, all) - 1) / all); }
template <int QB, int UNIT, bool PLAN> struct Walk {
  int id, part;                           // with a plan: the run; else tile and head (tile + head * tiles), and the range
  int64_t x, x1;                          // with a plan: units to do
  // of block `block`; all first ranges come first, then the second ones: the last to start are those that only the longest tiles have
  __device__ __forceinline__ Walk(const PagedArgs& a, int block) : Walk(a, PLAN ? block : block % (a.tiles * a.hk), PLAN ? 0 : block / (a.tiles * a.hk)) {}
  __device__ __forceinline__ Walk(const PagedArgs& a, int id_, int part_) : id(id_), part(part_), x(0), x1(0) {
    if constexpr (PLAN) {
      const int64_t all = (int64_t)uniform_i32(a.plan + a.tiles) * a.hk;
      if (id < runs_of(a, all)) {
        x = first_of(a, id, all);
        x1 = first_of(a, id + 1, all);
      }
    }
  }
  __device__ __forceinline__ bool next(const PagedArgs& a, Piece& p) {
    if constexpr (!PLAN) {                                    // one piece
      const int part = __builtin_amdgcn_readfirstlane(this->part);
      if (!locate<QB>(a, id % a.tiles, id / a.tiles, p.b)) return false;
      p.k0 = part * a.part_keys;
      p.k1 = p.b.end < p.k0 + a.part_keys || a.parts == 1 ? p.b.end : p.k0 + a.part_keys;
      p.slot = a.parts > 1 && p.b.end > a.part_keys ? __builtin_amdgcn_readfirstlane(id) * a.parts + part : -1;
      return p.k0 < p.k1 || part == 0;
    } else {
      if (x >= x1) return false;
      const int of_head = uniform_i32(a.plan + a.tiles), hk = (int)(x / of_head), r = (int)(x - (int64_t)hk * of_head), lane = threadIdx.x & 63;
      // the last tile that begins at r or before (those without units lie before it), 64 of them at a look
      int lo = 0, hi = a.tiles;
      while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, at = lo + lane * step;
        const int n = __popcll(__ballot(at < hi && a.plan[at < hi ? at : lo] <= r));
        lo += (n - 1) * step;
        hi = lo + step < hi ? lo + step : hi;
      }
      lo = __builtin_amdgcn_readfirstlane(lo);
      const int u0 = r - uniform_i32(a.plan + lo), units = uniform_i32(a.plan + lo + 1) - uniform_i32(a.plan + lo);
      const int n = units - u0 < x1 - x ? units - u0 : (int)(x1 - x);
      x += n;
      if (!locate<QB>(a, lo, hk, p.b)) return false;            // never: only sequences with new tokens have units
      p.k0 = __builtin_amdgcn_readfirstlane(u0 * UNIT);
      const int k1 = (u0 + n) * UNIT;
      p.k1 = __builtin_amdgcn_readfirstlane(k1 < p.b.end ? k1 : p.b.end);
      p.slot = __builtin_amdgcn_readfirstlane(u0 == 0 && n == units ? -1 : 2 * id + (u0 == 0));
      return true;
    }
  }
};
// what a row of the block sees; 0 beyond the sequence's rows
__device__ __forceinline__ int row_end(const PagedArgs& a, const Block& k, int row) {
  if (row >= k.rows) return 0;
  const int e = seen_keys(a, row / a.shared, k.s.n, k.s.keys);
  return e < k.held ? e : k.held;
}
// offset of a row of q or of the output, in elements; row < k.rows
__device__ __forceinline__ int64_t row_at(const PagedArgs& a, const Block& k, int row, int64_t ts, int64_t hs) {
  const int i = row / a.shared, g = row - i * a.shared;
  return (int64_t)(k.s.row0 + i) * ts + (int64_t)(k.hk * a.shared + g) * hs;
}
// Rows of the pages that hold keys key_of(0), key_of(1) .. (uniform) of the block's sequence and head, which sees a key at least (k.end > 0).  Beyond its last
// page the last one is taken again, for a page that does not exist the first: what is read there is masked.  All entries of the table are asked for
// before the first is looked at.
template <int G, typename KeyOf> __device__ __forceinline__ void page_rows(const PagedArgs& a, const Block& k, int64_t (&at)[G], KeyOf&& key_of) {
  const int last = (k.end - 1) >> a.page_shift;
  const int32_t* const table = a.table + (int64_t)k.b * a.table_width;
  int32_t page[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int p = key_of(g) >> a.page_shift;
    page[g] = uniform_i32(table + (p < last ? p : last));
  }
#pragma unroll
  for (int g = 0; g < G; ++g)
    at[g] = (((int64_t)((uint32_t)page[g] < (uint32_t)a.n_pages ? page[g] : 0) * 2 * a.hk + k.hk) << a.page_shift) + (key_of(g) & ((1 << a.page_shift) - 1));
}
// A tile of keys comes in N trips of W wavefronts, RW rows each (powers of two).  Pages hold whole groups of 16 keys, so trips that share such a group share a look
// at the table: `at` has the first row of each group, or where a trip takes 16 rows and more, this wavefront's first row of each trip.
template <int N, int W, int RW> struct TileRows {
  static constexpr int SHARE = W * RW >= 16 ? 1 : 16 / (W * RW) < N ? 16 / (W * RW) : N, G = N / SHARE;
  int64_t at[G];
  __device__ __forceinline__ void look(const PagedArgs& a, const Block& b, int key0, int w) {
    page_rows(a, b, at, [&](int g) __attribute__((always_inline)) { return SHARE == 1 ? key0 + (g * W + w) * RW : key0 + g * 16; });
  }
  __device__ __forceinline__ int64_t row(int i, int w) const { return SHARE == 1 ? at[i] : at[i / SHARE] + w * RW + i % SHARE * (W * RW); }
};
// whether the page of a key below k.end exists
__device__ __forceinline__ bool page_exists(const PagedArgs& a, const Block& k, int key) {
  return (uint32_t)a.table[(int64_t)k.b * a.table_width + (key >> a.page_shift)] < (uint32_t)a.n_pages;
}
// whether one of the pages of keys [k0, k1), k1 <= k.end, does not exist; called by all threads of a block
__device__ __forceinline__ bool pages_missing(const PagedArgs& a, const Block& k, int k0, int k1) {
  bool bad = false;
  const int p1 = (k1 - 1) >> a.page_shift;
  for (int p = (k0 >> a.page_shift) + (int)threadIdx.x; k1 > k0 && p <= p1; p += blockDim.x)
    bad |= (uint32_t)a.table[(int64_t)k.b * a.table_width + p] >= (uint32_t)a.n_pages;
  return __syncthreads_or(bad);
}

typedef float f32x4 __attribute__((ext_vector_type(4)));

// The softmax of 16 rows (one a lane & 15; the four lanes of a row hold keys of their own): reference and sums so far.  m is in units of
// log2, after the scale; -inf as long as there is no score above it.
struct Soft { float m, l; };

template <int KT> __device__ __forceinline__ float maximum(const f32x4 (&sc)[KT], int kt1) {
  float mx = -INFINITY;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
    if (kt < kt1)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[kt][r]);
  mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
  return fmaxf(mx, __shfl_xor(mx, 32, 64));
}
// raises the reference to the tile's maximum: returns the factor of what was summed so far, and the reference to weigh with
__device__ __forceinline__ float raise(Soft& z, float top, float& ref) {
  const float m = fmaxf(z.m, top);
  ref = m == -INFINITY ? 0.f : m;
  const float alpha = __builtin_amdgcn_exp2f(z.m - ref);     // 0 while there was no reference
  z.m = m;
  z.l *= alpha;
  return alpha;
}
// What is not finite among the values that a row sees reaches its result, however small the weight: weights are above 0 in exact numbers, unless the score is
// -inf.  So a sum that is not finite is kept where its factor is 0 in fp32, and where a loop leaves such a sum (0 * infinity is NaN as well) the keys are gone
// through once more, with the values of every tile looked at, as those of a tile with a border always are.
__device__ __forceinline__ f32x4 lowered(f32x4 v, float f) {
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = f == 0.f && !(fabsf(v[r]) < INFINITY) ? v[r] : v[r] * f;
  return v;
}
__device__ __forceinline__ bool finite(f32x4 v) { return fmaf(v[0], 0.f, v[1] * 0.f) + fmaf(v[2], 0.f, v[3] * 0.f) == 0.f; }
template <int DT, int NT> __device__ __forceinline__ bool finite(const f32x4 (&o)[DT][NT]) {
  f32x4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = fmaf(o[d][t][r], 0.f, x[r]);
  return finite(x);
}
// Of a lane's four keys in each tile of 16 from key0 on: bit kt where their page does not exist (pages hold whole groups of 16)
template <int KT> __device__ __forceinline__ uint32_t missing(const PagedArgs& a, const Block& b, int key0, int lane) {
  uint32_t gone = 0;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    const int key = key0 + kt * 16 + (lane >> 4) * 4;
    gone |= (page_exists(a, b, key < b.end ? key : b.end - 1) ? 0u : 1u) << kt;
  }
  return gone;
}
// -inf for the keys that a row does not see: key0 is the tile's first, end the row's border
template <int KT> __device__ __forceinline__ void hide(f32x4 (&sc)[KT], int key0, int end, uint32_t gone, int lane) {
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
#pragma unroll
    for (int r = 0; r < 4; ++r) sc[kt][r] = (key0 + kt * 16 + (lane >> 4) * 4 + r >= end) | ((gone >> kt) & 1) ? -INFINITY : sc[kt][r];
}
// 1 / l, or 0 for a row without a weight; NaN stays
__device__ __forceinline__ float inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float over_lanes(float v) { v += __shfl_xor(v, 16, 64); return v + __shfl_xor(v, 32, 64); }
// four channels of an output row
__device__ __forceinline__ void store_four(float* p, f32x4 v) { *(f32x4*)p = v; }
__device__ __forceinline__ void store_four(bf16_t* p, f32x4 v) { *(uint2*)p = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])); }

// A lane's channels of a row, of tiles of 16: tile d holds channels d * 16 .. (lane >> 4) * 4 + r of them in register r; SPREAD: channel row * (HD / 16) + d of
// row (lane >> 4) * 4 + r.
template <int HD, int NT, bool SPREAD> __device__ __forceinline__ void put_row(float* to, const f32x4 (&o)[HD / 16][NT], int t, int lg, float f) {
  if constexpr (SPREAD) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int d = 0; d < HD / 16; d += 4) *(f32x4*)(to + (lg * 4 + r) * (HD / 16) + d) = f32x4{o[d][t][r], o[d + 1][t][r], o[d + 2][t][r], o[d + 3][t][r]} * f;
  } else {
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) *(f32x4*)(to + d * 16 + lg * 4) = o[d][t] * f;
  }
}
// The end of a block whose W wavefronts have the same NT * 16 rows and keys of their own: joined 16 rows at a time, every wavefront's m and l and its
// O^T by rows, added up in wavefront order at the common reference.  smem: W * 16 * (2 + HD + 4) floats, which every wavefront is done with.
template <typename T, int HD, int NT, int W, bool SPREAD>
__device__ __forceinline__ void join_waves(const PagedArgs& a, const Block& b, float* smem, const Soft (&z)[NT], const f32x4 (&o)[HD / 16][NT], int slot, int wave, int lane) {
  constexpr int OS = HD + 4, QB = NT * 16;
  float* const ml = smem;                                    // [W][16][2]
  float* const os = ml + W * 16 * 2;                         // [W][16][OS]
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (b.first + t * 16 >= b.rows) break;
    __syncthreads();
    const float lsum = over_lanes(z[t].l);
    if (lane < 16) { ml[(wave * 16 + lane) * 2] = z[t].m; ml[(wave * 16 + lane) * 2 + 1] = lsum; }
    put_row<HD, NT, SPREAD>(os + (wave * 16 + (lane & 15)) * OS, o, t, lane >> 4, 1.f);
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * (HD / 4); i += W * 64) {
      const int r = i / (HD / 4), c = i % (HD / 4) * 4, row = t * 16 + r;
      if (b.first + row >= b.rows) continue;
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < W; ++w) m = fmaxf(m, ml[(w * 16 + r) * 2]);
      const float ref = m == -INFINITY ? 0.f : m;
      float l = 0.f;
      f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = __builtin_amdgcn_exp2f(ml[(w * 16 + r) * 2] - ref);
        l += ml[(w * 16 + r) * 2 + 1] * f;
        v += *(const f32x4*)(os + (w * 16 + r) * OS + c) * f;
      }
      if (!finite(v)) {
        v = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < W; ++w) v += lowered(*(const f32x4*)(os + (w * 16 + r) * OS + c), __builtin_amdgcn_exp2f(ml[(w * 16 + r) * 2] - ref));
      }
      if (slot < 0) {
        store_four((T*)a.out + row_at(a, b, b.first + row, a.o_ts, a.o_hs) + c, v * inverse(l));
      } else {
        float* const ps = a.partial + (size_t)slot * (QB * (2 + HD));
        if (c == 0) { ps[row] = m; ps[QB + row] = l; }
        *(f32x4*)(ps + 2 * QB + row * HD + c) = v;
      }
    }
  }
}

// Joins the partial results of a tile's rows: a lane has four channels of a row.  SPLIT groups of lanes deal a row's partial results out (8 where rows are
// few and results may be many: 235 of them took 45 us one behind the other, now 6) and meet in LDS, in their order.  12 heads of 1560 rows of 128 in three
// ranges: 9 us for 33 MB.
template <int HD, int SPLIT> struct Joined {
  static constexpr int LANES = HD / 4, ROWS = 256 / LANES / SPLIT;           // lanes of a row, rows of a block
  static __host__ __device__ __forceinline__ int blocks_of_tile(const PagedArgs& a, int qb) {
    const int64_t most = (int64_t)a.max_q * a.shared;
    return ((most < qb ? (int)most : qb) + ROWS - 1) / ROWS;
  }
};
template <typename T, int HD, int QB, int SPLIT>
__global__ __launch_bounds__(256) void k_paged_join(const PagedArgs a) {
  typedef Joined<HD, SPLIT> J;
  constexpr int LANES = J::LANES;
  __shared__ float ms[SPLIT > 1 ? 256 / LANES : 1], ls[SPLIT > 1 ? 256 / LANES : 1];
  __shared__ f32x4 vs[SPLIT > 1 ? 256 : 1];
  const int per = J::blocks_of_tile(a, QB), id = blockIdx.x / per, group = threadIdx.x / LANES, split = group % SPLIT;
  const int row = (int)(blockIdx.x % per) * J::ROWS + group / SPLIT, c = threadIdx.x % LANES * 4;
  Block b;
  if (!locate<QB>(a, id % a.tiles, id / a.tiles, b)) return;
  const bool mine = b.first + row < b.rows;
  int parts, first;                                          // partial results, and the slot of the first
  if (a.plan) {
    const int tile = id % a.tiles, of_head = uniform_i32(a.plan + a.tiles);
    const int64_t all = (int64_t)of_head * a.hk, x = (int64_t)(id / a.tiles) * of_head + uniform_i32(a.plan + tile);
    const int g = run_of(a, x, all);
    parts = run_of(a, (int64_t)(id / a.tiles) * of_head + uniform_i32(a.plan + tile + 1) - 1, all) - g + 1;
    first = 2 * g + 1;
  } else {
    parts = (int)(((int64_t)b.end + a.part_keys - 1) / a.part_keys);
    first = id * a.parts;
  }
  if (parts < 2) return;                                     // one block had all of it
  auto at = [&](int i) __attribute__((always_inline)) {
    return a.partial + (size_t)(a.plan && i > 0 ? first - 1 + 2 * i : first + i) * (QB * (2 + HD));
  };
  const int from = mine ? split : parts;
  float m = -INFINITY;
#pragma unroll 4
  for (int i = from; i < parts; i += SPLIT) m = fmaxf(m, at(i)[row]);
  if constexpr (SPLIT > 1) {
    if (c == 0) ms[group] = m;
    __syncthreads();
#pragma unroll
    for (int s = 0; s < SPLIT; ++s) m = fmaxf(m, ms[group - split + s]);
  }
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = from; i < parts; i += SPLIT) {
    const float* const p = at(i);
    const float f = __builtin_amdgcn_exp2f(p[row] - ref);
    l += p[QB + row] * f;
    v += *(const f32x4*)(p + 2 * QB + row * HD + c) * f;
  }
  if (!finite(v)) {
    v = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i = from; i < parts; i += SPLIT) v += lowered(*(const f32x4*)(at(i) + 2 * QB + row * HD + c), __builtin_amdgcn_exp2f(at(i)[row] - ref));
  }
  if constexpr (SPLIT > 1) {
    if (c == 0) ls[group] = l;
    vs[threadIdx.x] = v;
    __syncthreads();
    if (split > 0) return;
#pragma unroll
    for (int s = 1; s < SPLIT; ++s) {
      l += ls[group + s];
      v += vs[threadIdx.x + s * LANES];
    }
  }
  if (mine) store_four((T*)a.out + row_at(a, b, b.first + row, a.o_ts, a.o_hs) + c, v * inverse(l));
}
template <typename T, int HD, int QB> void launch_join(const PagedArgs& a, hipStream_t st) {
  constexpr int SPLIT = QB <= 32 ? 8 : 1;
  if (a.plan || a.parts > 1) k_paged_join<T, HD, QB, SPLIT><<<(unsigned)((int64_t)a.tiles * a.hk * Joined<HD, SPLIT>::blocks_of_tile(a, QB)), 256, 0, st>>>(a);
}

// ---- host: what a call takes
struct Route { int qb, parts, part_keys, runs; int64_t tiles, tiles_of_seq; };   // rows of a block, ranges of its keys, or runs of a plan
inline int64_t tiles_of_call(const PagedArgs& a, int qb) {
  const int64_t each = ((int64_t)a.max_q * a.shared + qb - 1) / qb, all = a.n_tokens * a.shared / qb + a.n_seqs;
  return each == 1 ? (int64_t)a.n_seqs : each * a.n_seqs < all ? each * a.n_seqs : all;
}
// A kind of block: its rows, the keys of a step, the steps that a range has at least, how many a CU holds, beside how many the longest of unequal blocks is taken
// to run at most, and in units of 10 ns a step with 1, 2 .. of them on a CU, and what is done around the steps.
struct Kind { int qb, keys, least, per_cu, beside; int64_t step[4], around; };
// The kind and the ranges by an estimate of the time.  One sequence, seen whole: rounds of equal blocks.  Sequences of several lengths and causal borders: all
// the work, with a little over half of the bound's keys on average, and half of the longest block at the end; at least that block.  Ranges cost a launch
// and their partial results, written and read at 4.2 TB/s, and a little for each that the estimate does not see.  Where blocks fill the chip many times over there
// are none, which bounds the workspace.
inline void choose(const PagedArgs& a, const Kind* kinds, int n_kinds, int head_dim, Route& r) {
  const bool even = a.n_seqs == 1 && a.group == 0;
  int64_t best = INT64_MAX;
  for (const Kind* k = kinds; k < kinds + n_kinds; ++k) {
    const int64_t n = tiles_of_call(a, k->qb), key_tiles = (a.max_kv + k->keys - 1) / k->keys, slots = k->per_cu * 256;
    for (int64_t parts = 1; parts <= 32; ++parts) {
      const int64_t blocks = n * a.hk * parts, steps = (key_tiles + parts - 1) / parts;
      if (parts > 1 && (steps < k->least || blocks > 16 * slots)) break;
      const int64_t full = steps * k->step[k->per_cu - 1] + k->around;
      int64_t cost = 0;
      if (even) {
        const int64_t last = blocks % slots;
        cost = blocks / slots * full + (last > 0 ? steps * k->step[(last - 1) / 256] + k->around : 0);
      } else {
        const int64_t on_cu = (blocks + 255) / 256, longest = steps * k->step[(on_cu < k->beside ? on_cu : k->beside) - 1] + k->around;
        cost = blocks * (steps * k->step[k->per_cu - 1] * 11 / 20 + k->around) / slots + steps * k->step[0] / 2;
        cost = cost > longest ? cost : longest;
      }
      if (parts > 1) cost += 775 + 25 * parts + blocks * k->qb * (head_dim + 2) * 8 / 42000;
      if (cost < best) { best = cost; r.qb = k->qb; r.tiles = n; r.parts = (int)parts; r.part_keys = (int)(steps * k->keys); }
    }
  }
}

// ---- what a call takes, the bytes of its workspace (partial results, then the plan), and the launches
inline size_t partial_bytes(const PagedArgs& a, const Route& r, int head_dim) {
  return (r.runs ? (size_t)r.runs * 2 : r.parts > 1 ? (size_t)r.tiles * a.hk * r.parts : 0) * r.qb * (2 + head_dim) * sizeof(float);
}
inline size_t workspace_bytes(const PagedArgs& a, const Route& r, int head_dim) {
  return partial_bytes(a, r, head_dim) + (r.runs ? ((size_t)r.tiles + 1) * sizeof(int32_t) : 0);
}
Route route_attn_paged_bf16(const PagedArgs& a, int head_dim, int format);
Route route_attn_paged_f32(const PagedArgs& a, int head_dim);
void launch_attn_paged_bf16(const PagedArgs& a, const Route& r, int head_dim, int format, hipStream_t st);
void launch_attn_paged_f32(const PagedArgs& a, const Route& r, int head_dim, int format, hipStream_t st);
