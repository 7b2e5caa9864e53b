// Attention of a chunk of new tokens over the pages of a key/value cache (dp_attn_paged).
//
// Simplest form: one wavefront per new token and query head, 64 keys at a time (a lane owns a key's score), online softmax in fp32, the weighted sum
// over the values with a lane owning channels.
#include <math.h>

#include "paged.h"

namespace {

struct PagedArgs {
  const void* data;
  const uint8_t* scales;
  const void* q;
  void* out;
  int64_t q_ts, q_hs, o_ts, o_hs, n_tokens;
  const int32_t *q_start, *kv_len, *table;
  int32_t n_pages, page_shift, hk, shared, n_seqs, max_q, max_kv, table_width, group;
  float scale;                            // of the scores, times log2(e): softmax in powers of two
};
// a sequence's new tokens and keys, whatever the arrays hold
struct Seq { int64_t row0; int n, rows, keys; };
__device__ __forceinline__ Seq sequence(const PagedArgs& a, int b) {
  Seq s;
  int64_t r0 = a.q_start[b], r1 = a.q_start[b + 1];
  r0 = r0 < 0 ? 0 : r0 > a.n_tokens ? a.n_tokens : r0;
  r1 = r1 < r0 ? r0 : r1 > a.n_tokens ? a.n_tokens : r1;
  s.row0 = r0;
  s.n = (int)(r1 - r0);
  s.rows = s.n < a.max_q ? s.n : a.max_q;
  s.keys = a.kv_len[b] < 0 ? 0 : a.kv_len[b];
  return s;
}
// keys that exist in the table and within the bound
__device__ __forceinline__ int held(const PagedArgs& a, int keys) {
  const int64_t most = (int64_t)a.table_width << a.page_shift;
  const int k = keys < a.max_kv ? keys : a.max_kv;
  return k < most ? k : (int)most;
}
// keys that the i-th of n new tokens sees, of keys
__device__ __forceinline__ int seen(const PagedArgs& a, int i, int n, int keys) {
  if (a.group == 0) return keys;
  const int64_t p = (int64_t)keys - n + i;
  if (p < 0) return 0;
  const int64_t end = (p / a.group + 1) * a.group;
  return end < keys ? (int)end : keys;
}

template <typename T, int HD, bool CODES>
__global__ __launch_bounds__(64) void k_attn_paged_plain(const PagedArgs a) {
  __shared__ float sq[HD];
  const int lane = threadIdx.x, b = blockIdx.z, head = blockIdx.y, i = blockIdx.x;
  const Seq s = sequence(a, b);
  if (i >= s.rows) return;
  const int keys = held(a, s.keys), hk = head / a.shared;
  int end = seen(a, i, s.n, s.keys);
  end = end < keys ? end : keys;
  const T* const q = (const T*)a.q + (s.row0 + i) * a.q_ts + head * a.q_hs;
  for (int c = lane; c < HD; c += 64) sq[c] = Elem<T>::ld(q + c);
  __syncthreads();
  auto value = [&](int64_t row, int c) __attribute__((always_inline)) {
    if constexpr (CODES) return fp8x4_to_f32(((const uint8_t*)a.data)[row * HD + c], __uint_as_float((uint32_t)a.scales[row] << 23)).x;
    else return Elem<T>::ld((const T*)a.data + row * HD + c);
  };
  float m = -INFINITY, l = 0.f, o[HD / 64] = {};
  for (int k0 = 0; k0 < end; k0 += 64) {
    const int key = k0 + lane;
    int64_t row = -1;
    if (key < end) {
      const int page = a.table[(int64_t)b * a.table_width + (key >> a.page_shift)];
      if (page >= 0 && page < a.n_pages) row = ((((int64_t)page * 2 * a.hk) + hk) << a.page_shift) + (key & ((1 << a.page_shift) - 1));
    }
    float score = -INFINITY;
    if (row >= 0) {
      score = 0.f;
      for (int c = 0; c < HD; ++c) score = fmaf(sq[c], value(row, c), score);
      score *= a.scale;
    }
    float top = score;
    for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
    const float now = fmaxf(m, top), ref = now == -INFINITY ? 0.f : now;
    const float alpha = exp2f(m - ref), w = exp2f(score - ref);
    m = now;
    l = l * alpha + wave_sum(w);
    for (int c = 0; c < HD / 64; ++c) o[c] *= alpha;
    for (int j = 0; j < 64; ++j) {
      const float wj = __shfl(w, j, 64);
      const int64_t rj = __shfl((long long)row, j, 64);
      if (rj < 0 || wj == 0.f) continue;
      for (int c = 0; c < HD / 64; ++c) o[c] = fmaf(wj, value(rj + ((int64_t)a.hk << a.page_shift), c * 64 + lane), o[c]);
    }
  }
  T* const out = (T*)a.out + (s.row0 + i) * a.o_ts + head * a.o_hs;
  for (int c = 0; c < HD / 64; ++c) Elem<T>::st(out + c * 64 + lane, l > 0.f || l != l ? o[c] / l : 0.f);
}

const char* why_not_attn(const dp_kv_cache* c, const dp_attn_config* cfg) {
  if (const char* why = why_not_cache(c)) return why;
  if (!cfg) return "null pointer";
  if (cfg->q_heads < 1 || cfg->q_heads > 1024 || cfg->q_heads % c->kv_heads) return "q_heads must be a multiple of kv_heads in [1, 1024]";
  if (cfg->n_seqs < 0 || cfg->n_seqs > 65535) return "n_seqs must be in [0, 65535]";
  if (cfg->max_q < 0 || cfg->max_q > (1 << 24)) return "max_q must be in [0, 2^24]";
  if (cfg->max_kv < 0 || cfg->max_kv > 0x7fffffff - 65536) return "max_kv must be in [0, 2^31 - 1 - 65536]";
  if (cfg->table_width < 0) return "table_width must not be negative";
  if (cfg->causal_group < 0) return "causal_group must not be negative";
  if (!(cfg->scale > 0.f && cfg->scale < INFINITY)) return "scale must be positive and finite";
  return nullptr;
}

}  // namespace

#define REFUSE_IF(expr) do { if (const char* why = (expr)) return refuse(entry, why); } while (0)

extern "C" size_t dp_attn_paged_workspace_bytes(const dp_kv_cache* c, const dp_attn_config* cfg) {
  if (const char* why = why_not_attn(c, cfg)) { refuse("dp_attn_paged_workspace_bytes", why); return 0; }
  return 0;
}

extern "C" int dp_attn_paged(const dp_kv_cache* c, const dp_attn_config* cfg, const dp_rows* q, int64_t n_tokens, const int32_t* q_start,
                             const int32_t* kv_len, const int32_t* page_table, const dp_rows* out, void* workspace, size_t workspace_bytes,
                             void* stream) {
  static const char entry[] = "dp_attn_paged";
  REFUSE_IF(why_not_attn(c, cfg));
  REFUSE_IF(n_tokens < 0 || n_tokens > (1 << 24) ? "n_tokens must be in [0, 2^24]" : nullptr);
  if (n_tokens == 0 || cfg->n_seqs == 0 || cfg->max_q == 0) return DP_OK;
  REFUSE_IF(!q_start || !kv_len || (!page_table && cfg->table_width > 0) ? "null pointer" : nullptr);
  REFUSE_IF(((uintptr_t)q_start | (uintptr_t)kv_len | (uintptr_t)page_table) & 3 ? "index arrays must be 4-byte aligned" : nullptr);
  REFUSE_IF(why_not_rows(q, n_tokens, cfg->q_heads, c->head_dim, c->dtype, false));
  REFUSE_IF(why_not_rows(out, n_tokens, cfg->q_heads, c->head_dim, c->dtype, true));
  PagedArgs a{};
  a.data = c->data; a.scales = c->scales; a.q = q->data; a.out = out->data;
  a.q_ts = q->token_stride; a.q_hs = q->head_stride; a.o_ts = out->token_stride; a.o_hs = out->head_stride;
  a.n_tokens = n_tokens; a.q_start = q_start; a.kv_len = kv_len; a.table = page_table;
  a.n_pages = c->n_pages; a.page_shift = __builtin_ctz((unsigned)c->page_tokens); a.hk = c->kv_heads; a.shared = cfg->q_heads / c->kv_heads;
  a.n_seqs = cfg->n_seqs; a.max_q = cfg->max_q; a.max_kv = cfg->max_kv; a.table_width = cfg->table_width; a.group = cfg->causal_group;
  a.scale = cfg->scale * 1.4426950408889634f;
  const dim3 grid((unsigned)(cfg->max_q < n_tokens ? cfg->max_q : n_tokens), (unsigned)cfg->q_heads, (unsigned)cfg->n_seqs);
  const hipStream_t st = (hipStream_t)stream;
  const bool codes = c->format == DP_KV_FP8;
  (void)hipGetLastError();
#define PLAIN(T, HD) do { if (codes) k_attn_paged_plain<T, HD, true><<<grid, 64, 0, st>>>(a); else k_attn_paged_plain<T, HD, false><<<grid, 64, 0, st>>>(a); } while (0)
  if (c->dtype == DP_BF16) { if (c->head_dim == 128) PLAIN(bf16_t, 128); else PLAIN(bf16_t, 64); }
  else { if (c->head_dim == 128) PLAIN(float, 128); else PLAIN(float, 64); }
#undef PLAIN
  if (hipGetLastError() != hipSuccess) return dp_set_error(DP_EHIP, "dp_attn_paged: the launch failed");
  return DP_OK;
}
