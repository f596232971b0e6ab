// Attention of query tokens over the pages listed for each, straight from the pool.
//
// Every query token and KV head is a unit with a list of pages; what the kernels of dd_cache_attn.cuh do for the tiles of a request
// in order, they do here for the tiles of the listed pages. What differs: a table entry is found through the list (two
// dependent loads for 32 tiles at a time), the first token of a tile travels with the tile, since the list says nothing about
// where it lies, and the places of the flat list are added up by the threads of a block together, since there may be many tokens.
#include "dd_cache_attn.cuh"

extern "C" size_t dd_cache_sparse_attn_workspace(int n_q_heads, int n_kv_heads, int head_dim) {
  if (ca_check_heads(n_q_heads, n_kv_heads, head_dim, 1)) return 0;
  return ca_size(head_dim, n_q_heads / n_kv_heads, ca_sm_count()).total();
}

extern "C" int dd_cache_sparse_attn(const dd_cache* cache, int n_tokens, const int* positions, const int* requests, const dd_rows* q,
                                    const int* idx, int k_pages, const dd_rows* out, float* out_lse, float scale, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  const char* who = "dd_cache_sparse_attn";
  DD_TRY(dd_check_cache(cache, who));
  if (n_tokens < 0) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: n_tokens is negative", who);
  if (!requests && n_tokens % cache->batch)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: without requests, n_tokens (%d) must be a multiple of batch (%d)", who, n_tokens, cache->batch);
  if (k_pages < 1) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: k_pages must be positive", who);
  if (!(scale >= 0.f) || scale > 3.4e38f) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: scale must be finite and not negative", who);
  if (n_tokens == 0) return DD_OK;
  DD_TRY(dd_check_rows(q, who, "q", cache->head_dim, n_tokens, false));
  DD_TRY(dd_check_rows(out, who, "out", cache->head_dim, n_tokens, true));
  if (const char* why = ca_check_heads(q->n_heads, cache->n_kv_heads, cache->head_dim, 1)) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: %s", who, why);
  if (out->n_heads != q->n_heads || out->dtype != q->dtype)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: q and out differ in heads or type", who);
  if ((cache->format == DD_CACHE_BF16 && q->dtype != DD_BF16) || (cache->format == DD_CACHE_FP16 && q->dtype != DD_FP16))
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: a 16-bit cache takes queries of its own type", who);
  const int device = dd_current_device();
  const char* data = nullptr;
  DD_TRY(dd_check_cache_memory(cache, who, device, false, &data, nullptr));
  DD_TRY(dd_check_ptr(positions, who, "positions", 4, device));
  if (requests) DD_TRY(dd_check_ptr(requests, who, "requests", 4, device));
  DD_TRY(dd_check_ptr(q->data, who, "q", 16, device));
  DD_TRY(dd_check_ptr(idx, who, "idx", 4, device));
  DD_TRY(dd_check_ptr(out->data, who, "out", 16, device));
  if (out_lse) DD_TRY(dd_check_ptr(out_lse, who, "out_lse", 4, device));
  DD_TRY(dd_check_ptr(workspace, who, "workspace", 16, device));
  ca_args a = {};
  a.G = q->n_heads / cache->n_kv_heads;
  a.n_rows = a.G;
  a.by_G = (uint32_t)((0x80000000ull + a.G - 1) / a.G);
  const int sms = ca_sm_count();
  const ca_sizes z = ca_size(cache->head_dim, a.n_rows, sms);
  if (workspace_bytes < z.total())
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: workspace holds %zu bytes, %zu needed", who, workspace_bytes, z.total());
  const int nt = ca_column_tiles(a.n_rows);
  a.c = dd_make_view(cache, data);
  a.q = (const char*)q->data;
  a.out = (char*)out->data;
  a.q_token_stride = q->token_stride * 2; a.q_head_stride = q->head_stride * 2;
  a.out_token_stride = out->token_stride * 2; a.out_head_stride = out->head_stride * 2;
  a.lse = out_lse;
  a.part_o = (float4*)workspace;
  a.part_ml = (float2*)((char*)workspace + z.part_o);
  a.desc = (int4*)((char*)workspace + z.part_o + z.part_ml);
  a.n_q_heads = q->n_heads;
  a.Tq = 1;
  a.batch = n_tokens;
  a.positions = positions;
  a.requests = requests;
  a.tokens_per_request = requests ? 1 : n_tokens / cache->batch;
  a.idx = idx;
  a.k_pages = k_pages;
  a.unit_tiles = (k_pages < cache->max_pages ? k_pages : cache->max_pages) * (cache->page_tokens / 16);
  a.row_tiles = (a.n_rows + nt * 8 - 1) / (nt * 8);
  a.scale_log2 = (float)((scale > 0.f ? (double)scale : 1.0 / sqrt((double)cache->head_dim)) * 1.4426950408889634);
  if ((long long)a.row_tiles * cache->n_kv_heads > 0x7fffffffLL / 64)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: too many heads", who);
  ca_plan p;
  switch (ca_format(cache->format, q->dtype)) {
    case 0: p = ca_pick_of<0, true>(cache->head_dim, nt); break;
    case 1: p = ca_pick_of<1, true>(cache->head_dim, nt); break;
    case 2: p = ca_pick_of<2, true>(cache->head_dim, nt); break;
    case 3: p = ca_pick_of<3, true>(cache->head_dim, nt); break;
    case 4: p = ca_pick_of<4, true>(cache->head_dim, nt); break;
    default: p = ca_pick_of<5, true>(cache->head_dim, nt); break;
  }
  const int blocks = sms * p.blocks_per_sm;
  const long long units = (long long)n_tokens * a.row_tiles * cache->n_kv_heads;
  a.cluster = ca_cluster_spread(units, a.unit_tiles, blocks);
  a.joins = !a.cluster && a.unit_tiles > CA_WHOLE;                    // else no unit can have been cut
  return ca_launch(who, a, p, units, blocks, nt, cache->head_dim, (cudaStream_t)stream);
}
