/* The calls of the paged cache that use much shared memory, before and after cudaDeviceReset: what the library was granted for its
 * kernels goes with the context, and has to be asked for again. Exit code 0 = every call ran both times. */
#include <cuda_runtime_api.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "dd.h"

#define CHECK_DD(expr)                                                                              \
  do {                                                                                              \
    int rc__ = (expr);                                                                              \
    if (rc__ != DD_OK) {                                                                            \
      fprintf(stderr, "%s -> %d (%s): %s\n", #expr, rc__, dd_strerror(rc__), dd_last_error_message(NULL)); \
      return 1;                                                                                     \
    }                                                                                               \
  } while (0)
#define CHECK_CUDA(expr)                                                        \
  do {                                                                          \
    cudaError_t e__ = (expr);                                                   \
    if (e__ != cudaSuccess) {                                                   \
      fprintf(stderr, "%s -> %s\n", #expr, cudaGetErrorString(e__));            \
      return 1;                                                                 \
    }                                                                           \
  } while (0)

enum { N = 64, HKV = 2, HQ = 8, D = 128, T = 16, P = 40, K = 8 };

static int all_calls(void) {
  const size_t page = dd_cache_page_bytes(DD_CACHE_BF16, T, D), rows = (size_t)N * HQ * D * 2;
  const size_t lm_bytes = (size_t)P * HKV * dd_cache_landmark_bytes(D);
  size_t ws_bytes = dd_cache_select_workspace(N, HKV, P), more = dd_cache_sparse_attn_workspace(N, HQ, HKV, D, K);
  void *pool, *q, *out, *landmarks, *ws;
  int *table, *ctx_len, *positions, *idx, h_table[P], h_pos[N], h_len = P * T, h_idx[K], i;
  if (more > ws_bytes) ws_bytes = more;
  more = dd_cache_decode_attn_workspace(HQ, HKV, D, 1);
  if (more > ws_bytes) ws_bytes = more;
  CHECK_CUDA(cudaMalloc(&pool, page * HKV * P));
  CHECK_CUDA(cudaMemset(pool, 0, page * HKV * P));
  CHECK_CUDA(cudaMalloc(&q, rows));
  CHECK_CUDA(cudaMemset(q, 0, rows));
  CHECK_CUDA(cudaMalloc(&out, rows));
  CHECK_CUDA(cudaMalloc(&landmarks, lm_bytes));
  CHECK_CUDA(cudaMemset(landmarks, 0, lm_bytes));
  CHECK_CUDA(cudaMalloc(&ws, ws_bytes));
  CHECK_CUDA(cudaMalloc((void**)&table, sizeof(h_table)));
  CHECK_CUDA(cudaMalloc((void**)&ctx_len, sizeof(h_len)));
  CHECK_CUDA(cudaMalloc((void**)&positions, sizeof(h_pos)));
  CHECK_CUDA(cudaMalloc((void**)&idx, sizeof(int) * N * HKV * K));
  for (i = 0; i < P; ++i) h_table[i] = i;
  for (i = 0; i < N; ++i) h_pos[i] = P * T - N + i;
  CHECK_CUDA(cudaMemcpy(table, h_table, sizeof(h_table), cudaMemcpyHostToDevice));
  CHECK_CUDA(cudaMemcpy(positions, h_pos, sizeof(h_pos), cudaMemcpyHostToDevice));
  CHECK_CUDA(cudaMemcpy(ctx_len, &h_len, sizeof(h_len), cudaMemcpyHostToDevice));
  dd_cache c;
  memset(&c, 0, sizeof(c));
  c.data = pool; c.format = DD_CACHE_BF16; c.n_kv_heads = HKV; c.head_dim = D; c.page_tokens = T; c.n_blocks = P;
  c.head_stride = (long long)page; c.block_stride = (long long)page * HKV;
  c.block_table = table; c.batch = 1; c.max_pages = P; c.table_stride = P;
  dd_rows rq = {q, DD_BF16, HQ, (long long)HQ * D, D}, ro = {out, DD_BF16, HQ, (long long)HQ * D, D};
  CHECK_DD(dd_cache_decode_attn(&c, 1, &rq, ctx_len, &ro, NULL, 0, 0.f, ws, ws_bytes, NULL));
  CHECK_DD(dd_cache_landmarks(&c, ctx_len, 0, landmarks, NULL));
  CHECK_DD(dd_cache_select(&c, N, positions, NULL, &rq, landmarks, K, 0, 1, idx, ws, ws_bytes, NULL));
  CHECK_DD(dd_cache_sparse_attn(&c, N, positions, NULL, &rq, idx, K, &ro, NULL, 0.f, ws, ws_bytes, NULL));
  CHECK_CUDA(cudaDeviceSynchronize());
  CHECK_CUDA(cudaMemcpy(h_idx, idx + (size_t)(N - 1) * HKV * K, sizeof(h_idx), cudaMemcpyDeviceToHost));
  for (i = 0; i < K; ++i)                       /* equal scores: the lowest pages and the token's own */
    if (h_idx[i] != (i < K - 1 ? i : P - 1)) {
      fprintf(stderr, "entry %d is page %d\n", i, h_idx[i]);
      return 1;
    }
  return 0;
}

int main(void) {
  if (all_calls()) return 1;
  CHECK_CUDA(cudaDeviceReset());
  if (all_calls()) return 1;
  puts("AFTER RESET OK");
  return 0;
}
