// Shared by the kernels of the paged key-value cache: rotary positions, writing, reading back and attention.
#pragma once

#include <cuda_fp16.h>

#include "dd_common.cuh"

// Checks that need no context. Every message names the argument; the text goes to the calling thread's error slot. What can
// be said without a device is checked first (dd_check_cache, dd_check_rows, dd_check_rope), the pointers after that.
int dd_current_device();
int dd_check_cache(const dd_cache* c, const char* who);
int dd_check_rows(const dd_rows* r, const char* who, const char* what, int head_dim, long long n_tokens, bool is_output);
int dd_check_rope(const dd_rope* r, const char* who, int head_dim);
int dd_check_cache_memory(const dd_cache* c, const char* who, int device, bool allow_host, const char** data_dev, bool* on_host);
int dd_check_ptr(const void* p, const char* who, const char* what, int align, int device);

#define DD_TRY(expr)                \
  do {                              \
    int rc__ = (expr);              \
    if (rc__ != DD_OK) return rc__; \
  } while (0)

// What a kernel needs to know of a cache.
struct dd_cache_view {
  char* data;
  long long block_stride, head_stride;   // bytes
  const int* table;
  long long table_stride;                // elements
  int* status;
  int n_blocks, n_kv_heads, batch, max_pages;
  int page_shift;                        // log2 of the tokens per page
};
dd_cache_view dd_make_view(const dd_cache* c, const char* data_dev);
// A launch whose failure is reported here and left behind nowhere (the runtime's last error is cleared).
int dd_launch(const char* who, const cudaLaunchConfig_t* cfg, const void* kernel, void** args);

static inline int dd_log2i(int x) { int s = 0; while ((1 << s) < x) ++s; return s; }

#ifdef __CUDACC__

// First error wins; never traps. `status` may be NULL.
__device__ __forceinline__ void dd_status(int* status, int detail) {
  if (status && atomicCAS(status, 0, DD_ERR_INDEX_RANGE) == 0) status[1] = detail;
}

__device__ __forceinline__ float dd_to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float dd_to_float(__half v) { return __half2float(v); }

template <typename T> __device__ __forceinline__ float2 dd_unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 dd_unpack2<__nv_bfloat16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 dd_unpack2<__half>(uint32_t w) {
  return __half22float2(*reinterpret_cast<__half2*>(&w));
}
template <typename T> __device__ __forceinline__ uint32_t dd_pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t dd_pack2<__nv_bfloat16>(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t dd_pack2<__half>(float lo, float hi) {
  __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

// Four e4m3 codes -> two half2 (exact: every e4m3 value is a half).
__device__ __forceinline__ void dd_e4m3x4_to_half(uint32_t codes, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(codes));
}
// Four values -> four e4m3 codes, round to nearest even. The caller keeps |v| <= 448; NaN gives the NaN code.
__device__ __forceinline__ uint32_t dd_float_to_e4m3x4(float v0, float v1, float v2, float v3) {
  uint32_t r;
  asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\t"
      "mov.b32 %0, {a, b};\n\t}"
      : "=r"(r) : "f"(v0), "f"(v1), "f"(v2), "f"(v3));
  return r;
}
// Exponent byte of a row whose largest finite magnitude is amax: the smallest e >= -127 with amax <= 448 * 2^e, plus 127.
// 448 = 1.75 * 2^8, so e is the magnitude's binade minus 8, plus one when its significand is above 1.75.
__device__ __forceinline__ int dd_e4m3_exponent_byte(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (e < -127 ? -127 : e) + 127;
}
__device__ __forceinline__ float dd_two_to_byte(int byte) {      // 2^(byte - 127), byte 0 included (a subnormal)
  return __uint_as_float(byte ? (uint32_t)byte << 23 : 0x00400000u);
}

// One warp brings 16 tokens of an e4m3 page in host memory to two runs of 16-bit rows: K codes at k_run, V codes at v_run
// (16 * D bytes each), this lane's exponent byte at `ex` (lanes 0-15 K, 16-31 V). The 4128 bytes of a page start anywhere in
// a 128-byte line, and a load instruction that straddles lines asks the host link for each part of a line by itself, so
// the loads are aligned to the lines (372 -> 339 us for 4096 pages; the two half-used stores per load do not matter at that
// rate). Not present: zeros.
template <typename T, int D>
__device__ __forceinline__ void dd_e4m3_tile_by_lines(const char* k_run, const char* v_run, const char* ex_at, bool present, char* dst_k, char* dst_v) {
  constexpr int NW = 16 * D / 512 + 1;             // aligned windows of 512 bytes that cover a run
  const int lane = threadIdx.x & 31;
  uint4 w[2][NW];
  int q[2], ex = 0;                                // this lane's first chunk of 16 codes of each run (may be negative)
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const char* run = kv ? v_run : k_run;
    q[kv] = lane - (int)(((uintptr_t)run & 127) >> 4);
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      w[kv][i] = make_uint4(0u, 0u, 0u, 0u);
      if (present && q[kv] + i * 32 >= 0 && q[kv] + i * 32 < D) w[kv][i] = dd_ld_stream(run + (q[kv] + i * 32) * 16);
    }
  }
  if (present) ex = *reinterpret_cast<const unsigned char*>(ex_at);
#pragma unroll
  for (int kv = 0; kv < 2; ++kv)
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const int at = q[kv] + i * 32;
      const float s = dd_two_to_byte(__shfl_sync(0xffffffffu, ex, kv * 16 + ((at < 0 ? 0 : at) * 16 / D & 15)));
      if (at >= 0 && at < D) {
        const uint32_t v4[4] = {w[kv][i].x, w[kv][i].y, w[kv][i].z, w[kv][i].w};
        uint32_t o[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t lo, hi;
          dd_e4m3x4_to_half(v4[k], lo, hi);
          const float2 u = dd_unpack2<__half>(lo), v = dd_unpack2<__half>(hi);
          o[2 * k] = dd_pack2<T>(u.x * s, u.y * s);  // exact for bf16 but for results below its smallest normal
          o[2 * k + 1] = dd_pack2<T>(v.x * s, v.y * s);
        }
        char* to = (kv ? dst_v : dst_k) + at * 32;
        dd_st_v4(to, make_uint4(o[0], o[1], o[2], o[3]));
        dd_st_v4(to + 16, make_uint4(o[4], o[5], o[6], o[7]));
      }
    }
}

#endif  // __CUDACC__
