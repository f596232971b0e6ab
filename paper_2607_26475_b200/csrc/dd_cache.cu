// The paged key-value cache: argument checks shared by its calls, and the kernel that reads pages back.
#include "dd_cache.cuh"

// ---------------------------------------------------------------------------------------------
// checks
// ---------------------------------------------------------------------------------------------
// The current device, or -1 where there is none: the checks that need no device come first then, and the pointer checks fail.
int dd_current_device() {
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess) {
    cudaGetLastError();
    return -1;
  }
  return device;
}

int dd_check_ptr(const void* p, const char* who, const char* what, int align, int device) {
  if (!p) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: %s is NULL", who, what);
  if (((uintptr_t)p) & (uintptr_t)(align - 1))
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: %s is not %d-byte aligned", who, what, align);
  cudaPointerAttributes a;
  cudaError_t e = cudaPointerGetAttributes(&a, p);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: %s: %s", who, what, cudaGetErrorString(e));
  }
  if (a.type != cudaMemoryTypeDevice && a.type != cudaMemoryTypeManaged)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: %s is not device memory", who, what);
  if (a.type == cudaMemoryTypeDevice && a.device != device)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: %s lives on device %d, the current one is %d", who, what, a.device, device);
  return DD_OK;
}

int dd_check_rows(const dd_rows* r, const char* who, const char* what, int head_dim, long long n_tokens, bool is_output) {
  if (!r) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: %s is NULL", who, what);
  if (r->dtype != DD_BF16 && r->dtype != DD_FP16) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: %s has an unknown dtype", who, what);
  if (r->n_heads < 1) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: %s has no heads", who, what);
  if (r->token_stride < 0 || r->head_stride < 0 || r->token_stride % 8 || r->head_stride % 8)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: strides of %s must be non-negative multiples of 8 elements", who, what);
  if (is_output) {
    // rows of an output must not meet: tokens behind all heads of the one before, or heads behind all tokens of the one before
    const bool tokens_apart = n_tokens < 2 || r->token_stride >= (long long)(r->n_heads - 1) * r->head_stride + head_dim;
    const bool heads_apart = r->n_heads < 2 || r->head_stride >= (n_tokens - 1) * r->token_stride + head_dim;
    if ((n_tokens > 1 && r->token_stride < head_dim) || (r->n_heads > 1 && r->head_stride < head_dim) || (!tokens_apart && !heads_apart))
      return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: rows of %s overlap", who, what);
  }
  if (!r->data) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: %s is NULL", who, what);
  return DD_OK;
}

extern "C" size_t dd_cache_page_bytes(int format, int page_tokens, int head_dim) {
  if (head_dim != 64 && head_dim != 128) return 0;
  if (page_tokens < 16 || page_tokens > 256 || (page_tokens & (page_tokens - 1))) return 0;
  if (format == DD_CACHE_BF16 || format == DD_CACHE_FP16) return (size_t)4 * page_tokens * head_dim;
  if (format == DD_CACHE_E4M3) return (size_t)2 * page_tokens * head_dim + 2 * page_tokens;
  return 0;
}

int dd_check_cache(const dd_cache* c, const char* who) {
  if (!c) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: cache is NULL", who);
  const long long page = (long long)dd_cache_page_bytes(c->format, c->page_tokens, c->head_dim);
  if (!page)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: format %d with %d tokens of %d elements a page is not supported "
                   "(head_dim 64 or 128, page_tokens 16, 32, 64, 128 or 256)", who, c->format, c->page_tokens, c->head_dim);
  if (c->n_kv_heads < 1 || c->n_blocks < 1 || c->batch < 1 || c->max_pages < 1)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: sizes of the cache must be positive", who);
  if ((long long)c->max_pages * c->page_tokens > 0x7fffffffLL - 16)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: max_pages * page_tokens does not fit 31 bits", who);
  if (c->table_stride < c->max_pages && c->batch > 1)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: table_stride is below max_pages", who);
  if (c->table_stride < 0) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: table_stride is negative", who);
  if (c->block_stride % 16 || c->head_stride % 16 || c->block_stride < 0 || c->head_stride < 0)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: page strides must be non-negative multiples of 16 bytes", who);
  if ((c->n_blocks > 1 && c->block_stride < page) || (c->n_kv_heads > 1 && c->head_stride < page))
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: pages of %lld bytes overlap", who, page);
  if (!c->data) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: cache->data is NULL", who);
  if (((uintptr_t)c->data) & 15) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: cache->data is not 16-byte aligned", who);
  if (!c->block_table) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: cache->block_table is NULL", who);
  return DD_OK;
}

int dd_check_cache_memory(const dd_cache* c, const char* who, int device, bool allow_host, const char** data_dev, bool* on_host) {
  DD_TRY(dd_check_ptr(c->block_table, who, "cache->block_table", 4, device));
  if (c->status) DD_TRY(dd_check_ptr(c->status, who, "cache->status", 4, device));
  cudaPointerAttributes a;
  cudaError_t e = cudaPointerGetAttributes(&a, c->data);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: cache->data: %s", who, cudaGetErrorString(e));
  }
  if (a.type == cudaMemoryTypeUnregistered)
    return dd_fail(nullptr, DD_ERR_NOT_PINNED, "%s: cache->data is pageable host memory; page-lock it (cudaHostAlloc / cudaHostRegister)", who);
  if (a.type == cudaMemoryTypeHost) {
    if (!allow_host) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: cache->data must be device memory", who);
    if (!a.devicePointer) return dd_fail(nullptr, DD_ERR_NOT_PINNED, "%s: cache->data is page-locked but not mapped into the device", who);
    *data_dev = (const char*)a.devicePointer;
    if (on_host) *on_host = true;
    return DD_OK;
  }
  if (a.type == cudaMemoryTypeDevice && a.device != device)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: cache->data lives on device %d, the current one is %d", who, a.device, device);
  *data_dev = (const char*)c->data;
  if (on_host) *on_host = false;
  return DD_OK;
}

int dd_launch(const char* who, const cudaLaunchConfig_t* cfg, const void* kernel, void** args) {
  const cudaError_t e = cudaLaunchKernelExC(cfg, kernel, args);
  if (e == cudaSuccess) return DD_OK;
  cudaGetLastError();
  return dd_fail(nullptr, DD_ERR_CUDA, "%s: launch: %s", who, cudaGetErrorString(e));
}

dd_cache_view dd_make_view(const dd_cache* c, const char* data_dev) {
  dd_cache_view v;
  v.data = const_cast<char*>(data_dev);
  v.block_stride = c->block_stride;
  v.head_stride = c->head_stride;
  v.table = c->block_table;
  v.table_stride = c->table_stride;
  v.status = c->status;
  v.n_blocks = c->n_blocks;
  v.n_kv_heads = c->n_kv_heads;
  v.batch = c->batch;
  v.max_pages = c->max_pages;
  v.page_shift = dd_log2i(c->page_tokens);
  return v;
}

// ---------------------------------------------------------------------------------------------
// reading pages back
// ---------------------------------------------------------------------------------------------
// One warp per 16 tokens of a page: K and V of a tile are two contiguous runs, read with loads that are all in flight before
// the first store (4 KiB a warp for e4m3 at head_dim 128, 8 KiB for 16-bit pages), and written as two contiguous runs of
// 16-bit rows. A lane takes as many elements per load as it writes in one 16-byte store, so that every load and store of a
// warp covers one contiguous piece: 8-byte loads for e4m3 (16-byte loads left two half-used stores: 44 against 34 us for
// 16384 pages). Bound: HBM, or the host link for a page-locked pool. The exponents of a tile are 16 bytes for K and 16 for V:
// one byte per lane in one load, handed out by shuffles. Measured on a B200: 8192 e4m3 pages of 16 x 128 14.9 us (6.8 TB/s of
// reads and writes, inputs partly in L2), 32768 pages 65 us (6.2 TB/s); 4096 pages from page-locked memory 339 us (49.9 GB/s of
// the 51 that kernel reads get there), 4096 bf16 pages 656 us (51.1 GB/s).
constexpr int CR_THREADS = 256;

// LINES: e4m3 pages in host memory, read by aligned lines (dd_e4m3_tile_by_lines).
template <int FMT, typename T, int D, bool LINES>
__global__ void __launch_bounds__(CR_THREADS) dd_cache_read_kernel(dd_cache_view c, const int* __restrict__ idx,
                                                                  char* __restrict__ out, int k_pages, long long n_tiles) {
  constexpr bool FP8 = FMT == DD_CACHE_E4M3;
  constexpr int ES = FP8 ? 1 : 2;
  constexpr int NL = 16 * D / 256;                     // loads (and stores) per lane for the K (or V) part of a tile
  const int lane = threadIdx.x & 31;
  const int page_tokens = 1 << c.page_shift, tile_shift = c.page_shift - 4;
  const long long n_warps = (long long)gridDim.x * (CR_THREADS / 32);
  dd_grid_dependency_wait();
  for (long long item = (long long)(threadIdx.x >> 5) * gridDim.x + blockIdx.x; item < n_tiles; item += n_warps) {
    const long long entry = item >> tile_shift;        // position in idx
    const int tile = (int)(item - (entry << tile_shift));
    const long long bg = (entry >> 31) == 0 ? (long long)((unsigned)entry / (unsigned)k_pages) : entry / k_pages;
    const int j = (int)(entry - bg * k_pages);
    const int b = (int)((unsigned)bg / (unsigned)c.n_kv_heads), g = (int)bg - b * c.n_kv_heads;
    const int p = idx[entry];
    int blk = -1;
    if (p < 0 || p >= c.max_pages) {
      if (lane == 0) dd_status(c.status, p);
    } else {
      blk = c.table[b * c.table_stride + p];
      if (blk < 0 || blk >= c.n_blocks) {
        if (lane == 0) dd_status(c.status, blk);
        blk = -1;
      }
    }
    // rows of the output: unit bg, half kv, page j, tile
    char* dst = out + (((bg * 2 * k_pages + j) << tile_shift) + tile) * (16LL * 2 * D);
    const long long v_off = ((long long)k_pages << tile_shift) * (16LL * 2 * D);
    if (LINES) {
      const char* page = c.data + (blk < 0 ? 0 : blk * c.block_stride + g * c.head_stride);
      const char* run = page + tile * 16 * D;
      dd_e4m3_tile_by_lines<T, D>(run, run + page_tokens * D, page + 2 * page_tokens * D + (lane >> 4) * page_tokens + tile * 16 + (lane & 15),
                                  blk >= 0, dst, dst + v_off);
      continue;
    }
    uint4 r[2][NL];                                    // e4m3: the first two words
    int ex = 0;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll
      for (int i = 0; i < NL; ++i) r[kv][i] = make_uint4(0u, 0u, 0u, 0u);
    if (blk >= 0) {
      const char* page = c.data + blk * c.block_stride + g * c.head_stride;
      const char* src = page + tile * (16 * D * ES) + lane * (8 * ES);
#pragma unroll
      for (int kv = 0; kv < 2; ++kv)
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const char* at = src + kv * page_tokens * D * ES + i * (256 * ES);
          if (FP8) {
            asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(r[kv][i].x), "=r"(r[kv][i].y) : "l"(at));
          } else {
            r[kv][i] = dd_ld_stream(at);
          }
        }
      if (FP8)
        ex = *reinterpret_cast<const unsigned char*>(page + 2 * page_tokens * D + (lane >> 4) * page_tokens + tile * 16 + (lane & 15));
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        char* to = dst + (kv ? v_off : 0) + i * 512 + lane * 16;
        if (!FP8) {
          dd_st_v4(to, r[kv][i]);
        } else {
          const float s = dd_two_to_byte(__shfl_sync(0xffffffffu, ex, kv * 16 + (i * 256 + lane * 8) / D));
          const uint32_t w[2] = {r[kv][i].x, r[kv][i].y};
          uint32_t o[4];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t lo, hi;
            dd_e4m3x4_to_half(w[q], lo, hi);
            const float2 u = dd_unpack2<__half>(lo), v = dd_unpack2<__half>(hi);
            o[2 * q] = dd_pack2<T>(u.x * s, u.y * s);  // exact for bf16 but for results below its smallest normal
            o[2 * q + 1] = dd_pack2<T>(v.x * s, v.y * s);
          }
          dd_st_v4(to, make_uint4(o[0], o[1], o[2], o[3]));
        }
      }
    }
  }
}

template <int D>
static const void* cr_kernel_of(int format, int dtype, bool on_host) {
  if (format != DD_CACHE_E4M3) return (const void*)dd_cache_read_kernel<DD_CACHE_BF16, __nv_bfloat16, D, false>;   // a copy of 16-bit words
  if (dtype == DD_BF16)
    return on_host ? (const void*)dd_cache_read_kernel<DD_CACHE_E4M3, __nv_bfloat16, D, true>
                   : (const void*)dd_cache_read_kernel<DD_CACHE_E4M3, __nv_bfloat16, D, false>;
  return on_host ? (const void*)dd_cache_read_kernel<DD_CACHE_E4M3, __half, D, true>
                 : (const void*)dd_cache_read_kernel<DD_CACHE_E4M3, __half, D, false>;
}

extern "C" int dd_cache_read(const dd_cache* cache, const int* idx, int k_pages, void* out, int out_dtype, void* stream) {
  const char* who = "dd_cache_read";
  DD_TRY(dd_check_cache(cache, who));
  if (k_pages < 0) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: k_pages is negative", who);
  if (out_dtype != DD_BF16 && out_dtype != DD_FP16) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: unknown out_dtype", who);
  if ((cache->format == DD_CACHE_BF16 && out_dtype != DD_BF16) || (cache->format == DD_CACHE_FP16 && out_dtype != DD_FP16))
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: a 16-bit cache is read in its own type", who);
  if (k_pages == 0) return DD_OK;
  const int device = dd_current_device();
  const char* data = nullptr;
  bool on_host = false;
  DD_TRY(dd_check_cache_memory(cache, who, device, true, &data, &on_host));
  DD_TRY(dd_check_ptr(idx, who, "idx", 4, device));
  DD_TRY(dd_check_ptr(out, who, "out", 16, device));
  long long n_tiles = (long long)cache->batch * cache->n_kv_heads * k_pages * (cache->page_tokens / 16);
  long long blocks = (n_tiles + CR_THREADS / 32 - 1) / (CR_THREADS / 32);
  if (on_host && blocks > 16) blocks = 16;             // as many as the host link needs; the other SMs stay free
  if (blocks > 0x7fffffffLL) blocks = 0x7fffffffLL;
  dd_cache_view v = dd_make_view(cache, data);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(CR_THREADS);
  cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute at;
  dd_pdl_attr(&at);
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  void* args[] = {&v, &idx, &out, &k_pages, &n_tiles};
  return dd_launch(who, &cfg, cache->head_dim == 128 ? cr_kernel_of<128>(cache->format, out_dtype, on_host)
                                                     : cr_kernel_of<64>(cache->format, out_dtype, on_host), args);
}
