// Attention of a chunk of new tokens over the pages of a key/value cache: the C entry (kernels:
// attn_paged_bf16.hip, attn_paged_f32.hip).
#include <math.h>

#include "attn_paged.h"

namespace {

constexpr float LOG2_E = 1.4426950408889634f;

const char* why_not_attn(const dp_kv_cache* c, const dp_attn_config* cfg) {
  if (const char* why = why_not_cache(c)) return why;
  if (!cfg) return "null pointer";
  if (cfg->q_heads < 1 || cfg->q_heads > 1024 || cfg->q_heads % c->kv_heads) return "q_heads must be a multiple of kv_heads in [1, 1024]";
  if (cfg->n_seqs < 0 || cfg->n_seqs > 65535) return "n_seqs must be in [0, 65535]";
  if ((int64_t)cfg->n_seqs * c->kv_heads > 1 << 21) return "n_seqs * kv_heads must be at most 2^21";
  if (cfg->max_q < 0 || cfg->max_q > (1 << 24)) return "max_q must be in [0, 2^24]";
  if (cfg->max_kv < 0 || cfg->max_kv > 0x7fffffff - 65536) return "max_kv must be in [0, 2^31 - 1 - 65536]";
  if (cfg->table_width < 0) return "table_width must not be negative";
  if (cfg->causal_group < 0) return "causal_group must not be negative";
  if (!(cfg->scale > 0.f && cfg->scale * LOG2_E < INFINITY)) return "scale must be positive, and finite times log2(e)";
  return nullptr;
}

PagedArgs arguments(const dp_kv_cache* c, const dp_attn_config* cfg, int64_t n_tokens) {
  PagedArgs a{};
  a.data = c->data; a.scales = c->scales; a.n_tokens = n_tokens;
  a.n_pages = c->n_pages; a.page_shift = __builtin_ctz((unsigned)c->page_tokens); a.hk = c->kv_heads; a.shared = cfg->q_heads / c->kv_heads;
  a.n_seqs = cfg->n_seqs; a.max_q = cfg->max_q < n_tokens ? cfg->max_q : (int32_t)n_tokens; a.table_width = cfg->table_width; a.group = cfg->causal_group;
  const int64_t most = (int64_t)cfg->table_width << a.page_shift;
  a.max_kv = cfg->max_kv < most ? cfg->max_kv : (int32_t)most;
  a.scale = cfg->scale * LOG2_E;
  return a;
}
// 2^29 rows in blocks of at most 4 threads a row, and a block of at most 512 threads begun for each sequence and key head: launches stay below 2^32 threads
const char* why_not_tokens(int64_t n, const dp_attn_config* cfg) {
  return n < 0 || n > (1 << 24) || n * cfg->q_heads > 1 << 29 ? "n_tokens must be in [0, 2^24], n_tokens * q_heads at most 2^29" : nullptr;
}
}  // namespace

extern "C" size_t dp_attn_paged_workspace_bytes(const dp_kv_cache* c, const dp_attn_config* cfg, int64_t n_tokens) {
  const char* why = why_not_attn(c, cfg);
  if (!why) why = why_not_tokens(n_tokens, cfg);
  if (why) { refuse("dp_attn_paged_workspace_bytes", why); return 0; }
  if (n_tokens == 0 || cfg->n_seqs == 0 || cfg->max_q == 0) return 0;
  const PagedArgs a = arguments(c, cfg, n_tokens);
  return workspace_bytes(a, c->dtype == DP_BF16 ? route_attn_paged_bf16(a, c->head_dim) : route_attn_paged_f32(a, c->head_dim), c->head_dim);
}

// for the tests, which state the kind of block that each of their calls is meant to reach: its rows, the ranges of the keys and the keys of one, the runs of a plan
extern "C" void dp_attn_paged_route(const dp_kv_cache* c, const dp_attn_config* cfg, int64_t n_tokens, int32_t* qb_parts_keys_runs) {
  const PagedArgs a = arguments(c, cfg, n_tokens);
  const Route r = c->dtype == DP_BF16 ? route_attn_paged_bf16(a, c->head_dim) : route_attn_paged_f32(a, c->head_dim);
  const int32_t v[4] = {r.qb, r.parts, r.part_keys, r.runs};
  for (int i = 0; i < 4; ++i) qb_parts_keys_runs[i] = v[i];
}

extern "C" int dp_attn_paged(const dp_kv_cache* c, const dp_attn_config* cfg, const dp_rows* q, int64_t n_tokens, const int32_t* q_start,
                             const int32_t* kv_len, const int32_t* page_table, const dp_rows* out, void* workspace, size_t have, void* stream) {
  static const char entry[] = "dp_attn_paged";
  REFUSE_IF(why_not_attn(c, cfg));
  REFUSE_IF(why_not_tokens(n_tokens, cfg));
  if (n_tokens == 0 || cfg->n_seqs == 0 || cfg->max_q == 0) return DP_OK;
  REFUSE_IF(!q_start || !kv_len || (!page_table && cfg->table_width > 0) ? "null pointer" : nullptr);
  REFUSE_IF(((uintptr_t)q_start | (uintptr_t)kv_len | (uintptr_t)page_table) & 3 ? "index arrays must be 4-byte aligned" : nullptr);
  REFUSE_IF(why_not_rows(q, n_tokens, cfg->q_heads, c->head_dim, c->dtype, false));
  REFUSE_IF(why_not_rows(out, n_tokens, cfg->q_heads, c->head_dim, c->dtype, true));
  PagedArgs a = arguments(c, cfg, n_tokens);
  a.q = q->data; a.out = out->data;
  a.q_ts = q->token_stride; a.q_hs = q->head_stride; a.o_ts = out->token_stride; a.o_hs = out->head_stride;
  a.q_start = q_start; a.kv_len = kv_len; a.table = page_table;
  const hipStream_t st = (hipStream_t)stream;
  const Route r = c->dtype == DP_BF16 ? route_attn_paged_bf16(a, c->head_dim) : route_attn_paged_f32(a, c->head_dim);
  a.tiles = (int32_t)r.tiles; a.tiles_of_seq = (int32_t)r.tiles_of_seq; a.parts = r.parts; a.part_keys = r.part_keys; a.runs = r.runs;
  if (const size_t need = workspace_bytes(a, r, c->head_dim)) {
    REFUSE_IF((uintptr_t)workspace & 255 ? "the workspace must be 256-byte aligned" : nullptr);
    if (!workspace || have < need) return dp_set_error(DP_ENOMEM, "dp_attn_paged: workspace too small");
    a.partial = (float*)workspace;
    if (r.runs) a.plan = (int32_t*)((char*)workspace + partial_bytes(a, r, c->head_dim));
  }
  (void)hipGetLastError();
  (c->dtype == DP_BF16 ? launch_attn_paged_bf16 : launch_attn_paged_f32)(a, r, c->head_dim, c->format == DP_KV_FP8, st);
  if (hipGetLastError() != hipSuccess) return dp_set_error(DP_EHIP, "dp_attn_paged: the launch failed");
  return DP_OK;
}
