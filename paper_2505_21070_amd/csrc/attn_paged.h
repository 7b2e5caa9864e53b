// What the attention kernels over a paged cache share: a call's arguments, which rows and keys a block of them owns, the way from a key
// to its row in the pages.
#pragma once
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
  // the launch: tiles of rows (of all sequences), the most a sequence has, ranges of keys a tile's work is cut into and keys of a range
  int32_t tiles, tiles_of_seq, parts, part_keys;
  float* partial;                         // parts > 1: [tile and head][part] of m[QB], l[QB], O[QB][head_dim]
};

// read through the scalar cache: uniform addresses of arrays that no kernel here writes
__device__ __forceinline__ int32_t uniform_i32(const int32_t* p) {
#ifdef __HIP_DEVICE_COMPILE__
  return *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)p;
#else
  return *p;
#endif
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

// The rows and keys of a block: tile `tile` of the call's tiles of QB rows, with key head `hk`.  Rows are (new token, shared head) pairs.
struct Block {
  int b, hk;                              // sequence, key head
  int first, rows;                        // its first row and one past the sequence's last
  Seq s;
  int held;                               // keys that exist for this sequence
  int end, whole;                         // keys that its last row sees, that its first row (and so every row) sees
};
// false: nothing to do.  Uniform; called by whole wavefronts.
template <int QB> __device__ __forceinline__ bool locate(const PagedArgs& a, int tile, int hk, Block& k) {
  int rb = 0;
  if (a.tiles_of_seq == 1) k.b = tile;
  else if (a.n_seqs == 1) { k.b = 0; rb = tile; }
  else {
    // tiles are numbered through the sequences: 64 of them at a time, a lane each
    const int lane = threadIdx.x & 63;
    int base = 0;
    k.b = -1;
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
        k.b = s0 + l;
        rb = tile - base - (__shfl(upto, l, 64) - __shfl(n, l, 64));
        break;
      }
      base += __shfl(upto, 63, 64);
    }
    if (k.b < 0) return false;
  }
  // what follows is the same in all lanes: kept in scalar registers, so that page tables are read through the scalar cache
  k.b = __builtin_amdgcn_readfirstlane(k.b);
  k.hk = __builtin_amdgcn_readfirstlane(hk);
  rb = __builtin_amdgcn_readfirstlane(rb);
  k.s = sequence(a, k.b);
  k.rows = k.s.rows * a.shared;
  // the last tile of a sequence first: under a causal border it has the most keys
  const int of_seq = (k.rows + QB - 1) / QB;
  if (rb >= of_seq) return false;
  k.first = __builtin_amdgcn_readfirstlane((of_seq - 1 - rb) * QB);
  k.held = held_keys(a, k.s.keys);
  const int last = (k.first + QB < k.rows ? k.first + QB : k.rows) - 1;
  const int e = seen_keys(a, last / a.shared, k.s.n, k.s.keys), w = seen_keys(a, k.first / a.shared, k.s.n, k.s.keys);
  k.end = __builtin_amdgcn_readfirstlane(e < k.held ? e : k.held);
  k.whole = __builtin_amdgcn_readfirstlane(w < k.held ? w : k.held);
  return true;
}
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
// Row of the pages that holds key `key` (uniform; at most 15 below a multiple of 16 that is not beyond key_end) of the block's sequence and head.  Beyond its last
// page the last one is taken again, for a page that does not exist the first: what is read there is masked.
__device__ __forceinline__ int64_t page_row(const PagedArgs& a, const Block& k, int key) {
  int at = key >> a.page_shift;
  const int last = (k.end - 1) >> a.page_shift;
  at = at < last ? at : last;
  const int page = uniform_i32(a.table + (int64_t)k.b * a.table_width + at);
  return (((int64_t)((uint32_t)page < (uint32_t)a.n_pages ? page : 0) * 2 * a.hk + k.hk) << a.page_shift) + (key & ((1 << a.page_shift) - 1));
}
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

// ---- the launches; each fills in the launch fields of a and returns the bytes of partial results it needs (partial == null: only that)
size_t launch_attn_paged_bf16(PagedArgs a, int head_dim, bool codes, bool go, hipStream_t st);
