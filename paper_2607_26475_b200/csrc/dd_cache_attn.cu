// Attention of the newest tokens of every request over all of its cached tokens (paged; 16-bit, e4m3 or 4-bit pages).
//
// Bound: HBM. Every K and V byte of the context is read once for every 16 query rows of its KV head (one row tile; beyond
// that once per row tile, 8 x 32K tokens bf16 with 24 rows 317 us against 178 with 16); 4 flops per element and row are far
// below the tensor peak. What has to be right is the load side: enough bytes in flight on every SM, no idle SM whatever the lengths
// are, and no pause at the border between two requests.
//
// Work split. The context of every (request, row tile, KV head) "unit" is cut into tiles of 16 tokens, and all tiles of
// the launch form one flat list, request by request, with a few empty places behind each unit that stand for what a unit
// costs besides its tiles. Every warp of a grid that fills the device once takes an equal run of the list; lengths are
// read on the device, so the launch does not depend on them (a captured graph may be replayed with other lengths). Units
// of at most 8 tiles are not cut. A warp works alone: it keeps a ring of half tiles (K or V) in flight with 16-byte
// cp.async, and the ring runs on across the borders of units. A copy instruction takes 512 contiguous bytes (whole 128-byte
// lines; fragments fetched straight from global memory touch half lines and ran at half the rate), and the chunks of a row are
// placed by row ^ chunk, so that ldmatrix reads them without bank conflicts: K as it lies, V transposed.
//
// Arithmetic, with the up-to-8 query rows of a KV head as the N = 8 columns of the MMA (two column tiles for up to 16
// rows, several row tiles beyond):
//   S^T[token, n] = K[token, :] . q[n, :]        A = K tile, B = q^T
//   O^T[d, n]    += V^T[d, token] P^T[token, n]   A = V^T, B = P^T
// e4m3 pages: codes are exact as halves, so both products run as half MMAs on the codes. The power-of-two scale of a key
// multiplies its scores; the scale of a value is added to the exponent of its weight: with w = z + log2(scale of v) the
// running reference is the maximum of w, P = 2^(w - ref) multiplies codes, and the denominator sums 2^(z - ref).
// The reference moves only when a weight exceeds it by 2^8 (one vote per tile instead of a reduction). Halves take a factor
// 2^6 that keeps small weights out of their subnormals (P at most 2^14; a weight 2^-20 of the reference is still normal),
// bf16 one of 2^-8 (P at most 1, as in a plain soft-max). Scales of e4m3 values from 2^-96 to 2^100 keep the denominator in
// range. Queries over e4m3 pages are multiplied by a power of two per row to fill the half's range: exact for every element
// above 2^-28 of the row's largest.
// 4-bit pages: the nibbles of a tile become halves in registers (ca_scale4): a nibble where it lies is a subnormal half, and one
// multiply-add makes (code - 8) * scale * 2^-17 of it, exactly. Pages are laid out for that: a lane's 16 bytes of K are 32 channels of one
// token (8 at head_dim 64: half of that), the MMA's slots take the channels in the order in which the nibbles come out, and the query rows are
// dealt to match; V lies by token pairs and eighths of the channels, so that a register's two halves are two tokens and nothing is transposed. Row
// exponents are used as for e4m3, the factor 2^17 comes back with the scores and at the end. A tile is copied whole, two complete ones are taken at a
// time. Per tile of 2336 bytes 350 instructions, of which 144 turn nibbles into halves. 8 x 32768 tokens are 47 us of bytes and 39 us of
// issue slots, and take 74.5: four warps a scheduler do not cover the latencies and the pipes' turns between the two.
//
// Rounding. A weight enters the second product as two 16-bit parts, its value cut off and the rounded rest (an MMA takes both
// operands in one type): off by 2^-16 relative at most for bf16 pages, by 2^-22 for half pages and half queries, so that the
// output's own rounding is the one that shows. One part (2^-8, 2^-11) left an error of 0.0023 relative on 4096 bf16 tokens where
// the output's rounding alone is 0.00165 (half: 0.00028 for 0.00021). The second part costs 168.1 -> 169.4 us on 8 x 32K tokens
// of bf16, 9.8 -> 10.1 us on 4096, and the same for half. e4m3 pages with bf16 queries go without: half weights (2^-11) are an
// eighth of the output's half step (0.00162 against 0.00161), and the part would cost 369 -> 375 us on 1M tokens; so do 4-bit pages with
// bf16 queries (errors of 0.00167 for 0.00166), where it would cost more: 8 x 32768 tokens 74 -> 84 us, 1M 241 -> 279, 48 ragged requests 60 -> 67, 2048
// tokens of 64 listed pages 596 -> 677. Halves end at
// 2^-24: a weight more than 2^31 below the reference is dropped, one above is off by 2^-31 of the reference at most. Queries as
// said, the output once. Scores, reference, denominators, accumulators and partial results are fp32.
//
// Joining. A unit inside one warp's run is finished there. The pieces of a cut unit that the warps of one block hold when
// their runs end are added in shared memory; what is left (one fp32 partial per block, and the unit's last piece) goes to
// the workspace, and a second small kernel adds those, always in the order of the list: the result does not depend on
// timing. Its blocks are launched early and wait for the first kernel's end. (Letting the last block of a unit to arrive do
// it, by a counter or by flags, took 4 to 7 us more: fences and contended words cost more round trips than a launch that
// is already there.)
//
// Measured on a B200 (device time of a call, 32 query and 8 KV heads of 128): 8 requests of 32768 tokens bf16 166-169 us
// (6.4 TB/s, a copy's rate), e4m3 105 us (5.2 TB/s; twice the instructions per byte, and four warps a scheduler do not cover
// their latencies), one request of 1M tokens e4m3 370-378 us (5.8 TB/s; 393 in passes that follow one another), 48 requests of 0
// to 32768 tokens e4m3 78-79 us, one request of 4096 tokens 10.0 us (13.2 where the table is 8192 pages wide). 4-bit pages: 8 x 32768 tokens
// (2 query tokens) 74.5 us (4.1 TB/s; 58% of the cycles issue), 1M tokens 242 us (5.1 TB/s), the ragged 48 60 us, 4096
// tokens 11.1 us, 100 tokens 7.9 us.
#include "dd_cache_attn.cuh"

extern "C" size_t dd_cache_decode_attn_workspace(int n_q_heads, int n_kv_heads, int head_dim, int n_q_tokens) {
  if (ca_check_heads(n_q_heads, n_kv_heads, head_dim, n_q_tokens)) return 0;
  return ca_size(head_dim, n_q_tokens * (n_q_heads / n_kv_heads), ca_sm_count()).total();
}

extern "C" int dd_cache_decode_attn(const dd_cache* cache, int n_q_tokens, const dd_rows* q, const int* ctx_len,
                                    const dd_rows* out, float* out_lse, int window, float scale, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  const char* who = "dd_cache_decode_attn";
  DD_TRY(dd_check_cache(cache, who));
  const long long n_tokens = (long long)cache->batch * n_q_tokens;
  DD_TRY(dd_check_rows(q, who, "q", cache->head_dim, n_tokens, false));
  DD_TRY(dd_check_rows(out, who, "out", cache->head_dim, n_tokens, true));
  if (const char* why = ca_check_heads(q->n_heads, cache->n_kv_heads, cache->head_dim, n_q_tokens))
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: %s", who, why);
  if (out->n_heads != q->n_heads || out->dtype != q->dtype)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: q and out differ in heads or type", who);
  if ((cache->format == DD_CACHE_BF16 && q->dtype != DD_BF16) || (cache->format == DD_CACHE_FP16 && q->dtype != DD_FP16))
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: a 16-bit cache takes queries of its own type", who);
  if (window < 0) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: window is negative", who);
  if (!(scale >= 0.f) || scale > 3.4e38f) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: scale must be finite and not negative", who);
  const int device = dd_current_device();
  const char* data = nullptr;
  DD_TRY(dd_check_cache_memory(cache, who, device, false, &data, nullptr));
  DD_TRY(dd_check_ptr(q->data, who, "q", 16, device));
  DD_TRY(dd_check_ptr(out->data, who, "out", 16, device));
  DD_TRY(dd_check_ptr(ctx_len, who, "ctx_len", 4, device));
  if (out_lse) DD_TRY(dd_check_ptr(out_lse, who, "out_lse", 4, device));
  DD_TRY(dd_check_ptr(workspace, who, "workspace", 16, device));
  const int sms = ca_sm_count();
  ca_args a = {};
  a.G = q->n_heads / cache->n_kv_heads;
  a.n_rows = n_q_tokens * a.G;
  a.by_G = (uint32_t)((0x80000000ull + a.G - 1) / a.G);
  const ca_sizes z = ca_size(cache->head_dim, a.n_rows, sms);
  if (workspace_bytes < z.total())
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: workspace holds %zu bytes, %zu needed", who, workspace_bytes, z.total());
  const int nt = ca_column_tiles(a.n_rows);
  a.c = dd_make_view(cache, data);
  a.q = (const char*)q->data;
  a.out = (char*)out->data;
  a.q_token_stride = q->token_stride * 2; a.q_head_stride = q->head_stride * 2;
  a.out_token_stride = out->token_stride * 2; a.out_head_stride = out->head_stride * 2;
  a.ctx_len = ctx_len;
  a.lse = out_lse;
  a.part_o = (float4*)workspace;
  a.part_ml = (float2*)((char*)workspace + z.part_o);
  a.desc = (int4*)((char*)workspace + z.part_o + z.part_ml);
  a.n_q_heads = q->n_heads;
  a.Tq = n_q_tokens;
  a.batch = cache->batch;
  a.unit_cost = ca_unit_cost(cache->format, false);
  a.row_tiles = (a.n_rows + nt * 8 - 1) / (nt * 8);
  a.window = window;
  a.scale_log2 = (float)((scale > 0.f ? (double)scale : 1.0 / sqrt((double)cache->head_dim)) * 1.4426950408889634);
  if ((long long)a.row_tiles * cache->n_kv_heads > 0x7fffffffLL / 64)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: too many heads", who);
  const ca_plan p = ca_pick<0>(ca_format(cache->format, q->dtype), cache->head_dim, nt);
  const int blocks = sms * p.blocks_per_sm;
  const long long units = (long long)cache->batch * a.row_tiles * cache->n_kv_heads;
  long long tiles = ((long long)cache->max_pages * cache->page_tokens + 15) / 16;
  if (window > 0 && ((long long)window + n_q_tokens + 29) / 16 < tiles) tiles = ((long long)window + n_q_tokens + 29) / 16;
  a.cluster = cache->format == DD_CACHE_INT4 ? ca_cluster_spread(units, tiles, blocks) : ca_cluster_of(units, tiles, blocks);
  a.joins = !a.cluster && (long long)cache->max_pages * cache->page_tokens > 16 * CA_WHOLE;   // else no unit can have been cut
  return ca_launch(who, a, p, units, blocks, nt, cache->head_dim, (cudaStream_t)stream);
}
