// Attention of query tokens over the pages listed for each, straight from the pool.
//
// Every query token and KV head is a unit with a list of pages; what the kernels of dd_cache_attn.cuh do for the tiles of a request
// in order, they do here for the tiles of the listed pages. What differs: a table entry is found through the list (two
// dependent loads for 32 tiles at a time), the first token of a tile travels with the tile, since the list says nothing about
// where it lies, and the places of the flat list are added up by the threads of a block together, since there may be many tokens.
#include "dd_cache_attn.cuh"

int dd_cache_pairs_launch(const char* who, ca_args& args, int format, int blocks, int head_dim, cudaStream_t stream);      // dd_cache_pairs.cu

namespace {

// ---- two tokens to a unit. Neighbouring tokens list many of the same pages, and the rows of one token fill the columns of an MMA by half or
// less (up to 4 query heads a KV head). The lists of tokens 2 i and 2 i + 1 are made one: a page that both list is read and
// multiplied once. Lists that ascend (as a selection gives them) of tokens of one request are merged by ranks; others are put one behind the other.
constexpr int CM_THREADS = 256;
constexpr int CM_MOST = 256;                           // entries of a list that is merged
struct cm_args {
  dd_cache_view c;
  const int* positions;
  const int* requests;
  const int* idx;
  int* merged;                                         // [pairs][heads][2 k]
  int* counts;                                         // [pairs]
  int n_tokens, tokens_per_request, k;
};
__global__ void __launch_bounds__(CM_THREADS) dd_cache_merge_kernel(const cm_args a) {
  __shared__ int sh_list[CM_THREADS / 32][2][CM_MOST];
  __shared__ int sh_most;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pair = blockIdx.x;
  dd_grid_dependency_wait();
  if (threadIdx.x == 0) sh_most = 0;
  __syncthreads();
  int own[2], req[2], seen[2];                         // own page, request, entries that are looked at
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const long long tok = 2LL * pair + i;
    own[i] = req[i] = -1;
    if (tok < a.n_tokens) {
      const int pos = a.positions[tok];
      req[i] = a.requests ? a.requests[tok] : (int)(tok / a.tokens_per_request);
      if (pos >= 0) {
        if ((unsigned)req[i] >= (unsigned)a.c.batch || (pos >> a.c.page_shift) >= a.c.max_pages) {
          if (threadIdx.x == 0) dd_status(a.c.status, (unsigned)req[i] >= (unsigned)a.c.batch ? req[i] : pos);
        } else {
          own[i] = pos >> a.c.page_shift;
        }
      }
    }
    seen[i] = min(a.k, own[i] + 1);
  }
  const unsigned below = (1u << lane) - 1u;
  for (int h = warp; h < a.c.n_kv_heads; h += CM_THREADS / 32) {
    int* const out = a.merged + ((long long)pair * a.c.n_kv_heads + h) * 2 * a.k;
    const int* const from[2] = {a.idx + (2LL * pair * a.c.n_kv_heads + h) * a.k, a.idx + ((2LL * pair + 1) * a.c.n_kv_heads + h) * a.k};
    bool ascending = own[0] >= 0 && own[1] >= 0 && req[0] == req[1] && a.k <= CM_MOST;
    int n[2] = {0, 0}, total = 0;
    __syncwarp();                                      // the lists of the head before have been read
    for (int i = 0; i < 2; ++i) {
      for (int j0 = 0; j0 < seen[i]; j0 += 32) {
        const int j = j0 + lane, p = j < seen[i] ? from[i][j] : -1;
        if (p < -1 || p >= a.c.max_pages) dd_status(a.c.status, p);
        const bool in = p >= 0 && p <= own[i];
        const unsigned all = __ballot_sync(0xffffffffu, in);
        // merged only where what is listed stands in front and ascends
        const bool good = !in || (j == n[i] + __popc(all & below) && (j == 0 || p > from[i][j - 1]));
        ascending = __all_sync(0xffffffffu, good) && ascending;
        if (ascending && in) sh_list[warp][i][j] = p;
        n[i] += __popc(all);
      }
    }
    if (ascending) {
      __syncwarp();
      auto lower = [&](const int* list, int m, int p) {               // entries below p
        int lo = 0;
        while (lo < m) {
          const int mid = (lo + m) / 2;
          if (list[mid] < p) lo = mid + 1;
          else m = mid;
        }
        return lo;
      };
      int both = 0;
      for (int i = 0; i < 2; ++i) {
        const int *mine = sh_list[warp][i], *other = sh_list[warp][1 - i];
        both = 0;                                      // pages of both lists in front
        for (int j0 = 0; j0 < n[i]; j0 += 32) {
          const int j = j0 + lane, p = j < n[i] ? mine[j] : -1, o = j < n[i] ? lower(other, n[1 - i], p) : 0;
          const bool common = j < n[i] && o < n[1 - i] && other[o] == p;
          const unsigned m = __ballot_sync(0xffffffffu, common);
          if (j < n[i] && (i == 0 || !common)) out[j + o - both - __popc(m & below)] = p | (common ? 3 : 1 + i) << 28;
          both += __popc(m);
        }
      }
      total = n[0] + n[1] - both;
    } else {
      for (int i = 0; i < 2; ++i)
        for (int j = lane; j < seen[i]; j += 32) {
          const int p = from[i][j];
          out[(i ? seen[0] : 0) + j] = p >= 0 && p <= own[i] ? p | (1 + i) << 28 : -1;
        }
      total = seen[0] + seen[1];
    }
    for (int j = total + lane; j < 2 * a.k; j += 32) out[j] = -1;
    if (own[0] >= 0 || own[1] >= 0) total = max(total, 1);            // somebody's rows are to be written
    if (lane == 0) atomicMax(&sh_most, total);
  }
  __syncthreads();
  if (threadIdx.x == 0) a.counts[pair] = sh_most;
}

// Pairs where they leave enough units to fill the device, two tokens a request and more, and both fit a column tile. Tokens of 64 pages of 32K, 8 KV
// heads of 4, us without | with pairs: bf16 pages 64 tokens 46 | 48, 200 112 | 93, 400 209 | 155, 800 336 | 259; 4-bit pages, whose tiles are worked
// on longer than they are brought, 64 42 | 49, 200 99 | 94, 400 159 | 163, 800 264 | 268. (16-bit pages would pay from half the bound on.)
bool cm_pairs(long long n_tokens, int batch, int n_kv_heads, int group, int sms) {
  return group <= 4 && n_tokens / batch >= 2 && n_tokens / 2 * n_kv_heads >= 8LL * sms;
}
size_t cm_bytes(long long n_tokens, int n_kv_heads, int k_pages) {
  const long long pairs = (n_tokens + 1) / 2;
  return (size_t)(pairs * n_kv_heads * 2 * k_pages * 4 + 15) / 16 * 16 + (size_t)(pairs * 4 + 15) / 16 * 16;
}

}  // namespace

extern "C" size_t dd_cache_sparse_attn_workspace(int n_tokens, int n_q_heads, int n_kv_heads, int head_dim, int k_pages) {
  if (ca_check_heads(n_q_heads, n_kv_heads, head_dim, 1) || n_tokens < 1 || k_pages < 1) return 0;
  const int sms = ca_sm_count(), group = n_q_heads / n_kv_heads;
  return ca_size(head_dim, group, sms).total() + (cm_pairs(n_tokens, 1, n_kv_heads, group, sms) ? cm_bytes(n_tokens, n_kv_heads, k_pages) : 0);
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
  if (k_pages > 0x3fffffff) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: k_pages is too large", who);
  ca_args a = {};
  a.G = q->n_heads / cache->n_kv_heads;
  a.n_rows = a.G;
  a.by_G = (uint32_t)((0x80000000ull + a.G - 1) / a.G);
  const int sms = ca_sm_count();
  const ca_sizes z = ca_size(cache->head_dim, a.n_rows, sms);
  const size_t need = dd_cache_sparse_attn_workspace(n_tokens, q->n_heads, cache->n_kv_heads, cache->head_dim, k_pages);
  if (workspace_bytes < need)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: workspace holds %zu bytes, %zu needed", who, workspace_bytes, need);
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
  a.unit_cost = ca_unit_cost(cache->format, true);
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
  const ca_plan p = ca_pick<1>(ca_format(cache->format, q->dtype), cache->head_dim, nt);
  const int blocks = sms * p.blocks_per_sm;
  a.n_tokens = n_tokens;
  if (cm_pairs(n_tokens, cache->batch, cache->n_kv_heads, a.G, sms)) {
    cm_args m = {};
    const int pairs = (n_tokens + 1) / 2;
    m.c = a.c;
    m.positions = positions;
    m.requests = requests;
    m.idx = idx;
    m.merged = (int*)((char*)workspace + z.total());
    m.counts = (int*)((char*)m.merged + ((size_t)pairs * cache->n_kv_heads * 2 * k_pages * 4 + 15) / 16 * 16);
    m.n_tokens = n_tokens;
    m.tokens_per_request = a.tokens_per_request;
    m.k = k_pages;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at;
    dd_pdl_attr(&at);
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    cfg.stream = (cudaStream_t)stream;
    cfg.gridDim = dim3((unsigned)pairs);
    cfg.blockDim = dim3(CM_THREADS);
    void* args[] = {&m};
    DD_TRY(dd_launch(who, &cfg, (const void*)dd_cache_merge_kernel, args));
    a.Tq = 2;
    a.batch = pairs;
    a.n_rows = 2 * a.G;
    a.idx = m.merged;
    a.counts = m.counts;
    a.k_pages = 2 * k_pages;
    a.joins = 1;
    return dd_cache_pairs_launch(who, a, ca_format(cache->format, q->dtype), blocks, cache->head_dim, (cudaStream_t)stream);
  }
  const long long units = (long long)n_tokens * a.row_tiles * cache->n_kv_heads;
  a.cluster = ca_cluster_spread(units, a.unit_tiles, blocks);
  a.joins = !a.cluster && a.unit_tiles > CA_WHOLE;                    // else no unit can have been cut
  return ca_launch(who, a, p, units, blocks, nt, cache->head_dim, (cudaStream_t)stream);
}
