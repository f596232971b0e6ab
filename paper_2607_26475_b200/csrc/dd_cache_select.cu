// Landmarks of a paged cache's pages, and the pages that each query token attends to.
//
// Landmark of (block, KV head): the mean of the page's keys as whole numbers l up to 127 times 2^e. Score of a page for query token n and
// KV head g: <c, l> * 2^e, c the sum of the group's query rows as whole numbers up to 127 (their power of two is the same for all pages of a row
// and left out). Sums and means are taken in 64 bits, where 16-bit values add up without a rounding for all but the wildest
// exponents; the product of whole numbers below 2^21 is exact whatever its order, and the power of two is exact in fp32. So the scores,
// and with them the chosen set, are defined to the last bit. (Adding up the group's rows orders pages as the product of the heads'
// soft-max probabilities does: what a head's soft-max divides by is the same for all pages.)
//
// Scores: whole-number MMAs, 16 pages as rows and 8 query tokens as columns. Few tokens a request: a block per token, which reads each landmark once (HBM
// bound: 144 bytes a page and head); many: 64 tokens of a head stay in registers while the pages go by. The keys (scores
// in an order that compares as unsigned numbers) of a bounded number of tokens go through a workspace that L2 holds.
//
// Choice: the k-th largest key by bisection, with the row's keys in registers: a step counts keys at or above the middle. It stops as
// soon as exactly k are (about a dozen steps for a few thousand keys); all the steps come up only with ties, which go to the lower pages.
#include "dd_cache.cuh"

namespace {

// ---- 64-bit rows as whole numbers
__device__ __forceinline__ double cs_finite(double v) { return fabs(v) <= 1.7976931348623157e308 ? v : 0.0; }
// The smallest e in [least, 63] with top <= 127 * 2^e (top finite, not negative): 127 = 1.984375 * 2^6.
__device__ __forceinline__ int cs_exponent(double top, int least) {
  const int hi = __double2hiint(top), lo = __double2loint(top);
  const int frac = hi & 0xfffff;
  const int e = ((hi >> 20) & 0x7ff) - 1023 - 6 + (frac > 0xfc000 || (frac == 0xfc000 && lo != 0) ? 1 : 0);
  return min(63, max(e, least));
}
__device__ __forceinline__ double cs_two_to(int e) { return __hiloint2double((e + 1023) << 20, 0); }
__device__ __forceinline__ int cs_code(double v, double down) { return (int)fmin(fmax(rint(v * down), -127.0), 127.0); }
__device__ __forceinline__ double cs_warp_max(double v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
constexpr int CS_TAIL = 16;                            // bytes behind the codes of a landmark: the exponent + 64, then nothing
constexpr int CS_LM_LEAST = -64, CS_Q_LEAST = -120;

// ---- landmarks: one warp per page and head, D / 32 channels a lane
constexpr int CL_THREADS = 256;
template <int FMT, int D>
__global__ void __launch_bounds__(CL_THREADS) dd_cache_landmark_kernel(dd_cache_view c, const int* __restrict__ ctx_len, int n_last, int pages, char* landmarks) {
  constexpr int N = D / 32;
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * (CL_THREADS / 32) + (threadIdx.x >> 5);
  const long long bp = item / c.n_kv_heads;
  const int h = (int)(item - bp * c.n_kv_heads), b = (int)(bp / pages);
  dd_grid_dependency_wait();
  if (b >= c.batch) return;
  int len = ctx_len[b];
  const int most = c.max_pages << c.page_shift;
  if (len < 0 || len > most) {
    if (lane == 0) dd_status(c.status, len);
    len = len < 0 ? 0 : most;
  }
  const int from = n_last > 0 && n_last < len ? len - n_last : 0;
  const long long p_ = (from >> c.page_shift) + (bp - (long long)b * pages);
  if ((p_ << c.page_shift) >= len) return;
  const int p = (int)p_, n = min(len - (p << c.page_shift), 1 << c.page_shift), T = 1 << c.page_shift;
  const int blk = c.table[b * c.table_stride + p];
  if ((unsigned)blk >= (unsigned)c.n_blocks) {
    if (lane == 0) dd_status(c.status, blk);
    return;
  }
  const char* page = c.data + blk * c.block_stride + h * c.head_stride;
  double sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = 0.0;
#pragma unroll 8
  for (int t = 0; t < n; ++t) {
    float v[N];
    if (FMT == DD_CACHE_INT4) {
      const char* tile = page + (t >> 4) * dd_int4_tile_bytes(D);
      const int r = t & 15;
      const uint32_t w = N == 4 ? *reinterpret_cast<const unsigned short*>(tile + r * (D / 2) + lane * 2) : *reinterpret_cast<const unsigned char*>(tile + r * (D / 2) + lane);
      uint32_t s2, unused;
      dd_e4m3x4_to_half(*reinterpret_cast<const unsigned char*>(tile + dd_int4_ks_at<D>(r, lane * N / 16)), s2, unused);
      const float s = dd_unpack2<__half>(s2).x, by = dd_two_to_byte(*reinterpret_cast<const unsigned char*>(tile + 18 * D + r));
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = (float)((int)(w >> (4 * i) & 15u) - 8) * s * by;
    } else if (FMT == DD_CACHE_E4M3) {
      const uint32_t w = N == 4 ? *reinterpret_cast<const uint32_t*>(page + t * D + lane * 4) : *reinterpret_cast<const unsigned short*>(page + t * D + lane * 2);
      const float by = dd_two_to_byte(*reinterpret_cast<const unsigned char*>(page + 2 * T * D + t));
      uint32_t lo, hi;
      dd_e4m3x4_to_half(w, lo, hi);
      const float2 x = dd_unpack2<__half>(lo), y = dd_unpack2<__half>(hi);
      v[0] = x.x * by;
      v[1] = x.y * by;
      if (N == 4) { v[N - 2] = y.x * by; v[N - 1] = y.y * by; }
    } else {
      uint2 w = make_uint2(0u, 0u);
      if (N == 4) w = *reinterpret_cast<const uint2*>(page + t * (2 * D) + lane * 8);
      else w.x = *reinterpret_cast<const uint32_t*>(page + t * (2 * D) + lane * 4);
      const float2 x = FMT == DD_CACHE_BF16 ? dd_unpack2<__nv_bfloat16>(w.x) : dd_unpack2<__half>(w.x);
      const float2 y = FMT == DD_CACHE_BF16 ? dd_unpack2<__nv_bfloat16>(w.y) : dd_unpack2<__half>(w.y);
      v[0] = x.x;
      v[1] = x.y;
      if (N == 4) { v[N - 2] = y.x; v[N - 1] = y.y; }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] += (double)v[i];
  }
  double top = 0.0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    sum[i] = cs_finite(sum[i] / (double)n);
    top = fmax(top, fabs(sum[i]));
  }
  const int e = cs_exponent(cs_warp_max(top), CS_LM_LEAST);
  const double down = cs_two_to(-e);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) w |= (uint32_t)(cs_code(sum[i], down) & 0xff) << (8 * i);
  char* to = landmarks + ((long long)blk * c.n_kv_heads + h) * (D + CS_TAIL);
  if (N == 4) *reinterpret_cast<uint32_t*>(to + lane * 4) = w;
  else *reinterpret_cast<unsigned short*>(to + lane * 2) = (unsigned short)w;
  if (lane < CS_TAIL / 4) *reinterpret_cast<uint32_t*>(to + D + lane * 4) = lane == 0 ? (uint32_t)(e + 64) : 0u;
}

// ---- scores
constexpr int CS_THREADS = 128;
struct cs_args {
  dd_cache_view c;
  const char* q;
  long long q_token_stride, q_head_stride;             // bytes
  const char* landmarks;
  const int* positions;
  const int* requests;
  uint32_t* keys;                                      // [tokens of the launch][heads][stride]
  int* out;
  int first_token, n_tokens, tokens_per_request;       // tokens first_token .. first_token + n_tokens - 1
  int G, k, first, recent;
  int stride;                                          // keys of a row
  int chunks, chunk_pages;                             // blocks that share a token tile, and how many pages each takes
};

// Own page of a token, -1 for padding and for one that names no place.
__device__ __forceinline__ int cs_own_page(const cs_args& a, int n, int& req, bool report) {
  const int pos = a.positions[n];
  req = a.requests ? a.requests[n] : n / a.tokens_per_request;
  if (pos < 0) return -1;
  const int own = pos >> a.c.page_shift;
  if ((unsigned)req >= (unsigned)a.c.batch || own >= a.c.max_pages) {
    if (report) dd_status(a.c.status, (unsigned)req >= (unsigned)a.c.batch ? req : pos);
    return -1;
  }
  return own;
}
// Order of scores as unsigned numbers.
__device__ __forceinline__ uint32_t cs_key(float z) {
  const uint32_t b = __float_as_uint(z);
  return b ^ ((int)b < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float cs_score(uint32_t key) { return __uint_as_float(key ^ ((int)key < 0 ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ void cs_mma(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// TT tokens of one head and a run of pages. Channels are dealt to the MMA's slots as they lie: lane t of a group of four takes the
// D / 4 channels from D / 4 t on, of landmarks and queries alike.
template <typename T, int D, int TT>
__global__ void __launch_bounds__(CS_THREADS) dd_cache_score_kernel(const cs_args a) {
  constexpr int CT = (TT + 7) / 8, N = D / 32;
  __shared__ __align__(16) unsigned char sh_q[CT * 8][D];
  __shared__ int sh_own[CT * 8], sh_req[CT * 8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int tile = blockIdx.x / a.chunks, chunk = blockIdx.x - tile * a.chunks, h = blockIdx.y;
  const int n0 = tile * TT;                            // of the launch
  dd_grid_dependency_wait();
  if (threadIdx.x < CT * 8) {
    int req = -1, own = -1;
    if (threadIdx.x < TT && n0 + threadIdx.x < a.n_tokens) own = cs_own_page(a, a.first_token + n0 + threadIdx.x, req, chunk == 0 && h == 0);
    sh_own[threadIdx.x] = own;
    sh_req[threadIdx.x] = req;
  }
  for (int i = warp; i < CT * 8; i += CS_THREADS / 32) {
    double sum[N];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0.0;
    if (i < TT && n0 + i < a.n_tokens) {
      const char* at = a.q + (a.first_token + n0 + i) * a.q_token_stride + (long long)h * a.G * a.q_head_stride + lane * (2 * N);
#pragma unroll 4
      for (int j = 0; j < a.G; ++j) {
        uint2 w = make_uint2(0u, 0u);
        if (N == 4) w = *reinterpret_cast<const uint2*>(at + j * a.q_head_stride);
        else w.x = *reinterpret_cast<const uint32_t*>(at + j * a.q_head_stride);
        const float2 x = dd_unpack2<T>(w.x), y = dd_unpack2<T>(w.y);
        sum[0] += (double)x.x;
        sum[1] += (double)x.y;
        if (N == 4) { sum[N - 2] += (double)y.x; sum[N - 1] += (double)y.y; }
      }
    }
    double top = 0.0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      sum[e] = cs_finite(sum[e]);
      top = fmax(top, fabs(sum[e]));
    }
    // (a sum of fp32-sized values stays below 2^64 * 127 only for those; larger ones are held at the largest number)
    const double down = cs_two_to(-cs_exponent(cs_warp_max(top), CS_Q_LEAST));
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) w |= (uint32_t)(cs_code(sum[e], down) & 0xff) << (8 * e);
    if (N == 4) *reinterpret_cast<uint32_t*>(&sh_q[i][lane * 4]) = w;
    else *reinterpret_cast<unsigned short*>(&sh_q[i][lane * 2]) = (unsigned short)w;
  }
  __syncthreads();
  uint32_t qf[CT][D / 16];                             // of token 8 ct + g: the words of this lane's channels
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const uint4 v = *reinterpret_cast<const uint4*>(&sh_q[ct * 8 + g][t * (D / 4) + i * 16]);
      qf[ct][4 * i] = v.x; qf[ct][4 * i + 1] = v.y; qf[ct][4 * i + 2] = v.z; qf[ct][4 * i + 3] = v.w;
    }
  const int p_begin = chunk * a.chunk_pages, p_end = min(p_begin + a.chunk_pages, a.c.max_pages);
  // tokens of one request at a time: tokens s .. e - 1 of the tile
  for (int s = 0, e; s < TT; s = e) {
    const int req = sh_req[s];
    int most = sh_own[s];
    for (e = s + 1; e < TT && sh_req[e] == req; ++e) most = max(most, sh_own[e]);
    if (most < 0) continue;
    const int* table = a.c.table + req * a.c.table_stride;
    const int last = min(p_end, most + 1);
    for (int p0 = p_begin + warp * 16; p0 < last; p0 += CS_THREADS / 2) {
      uint32_t r[2][D / 16];
      float by[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int p = p0 + g + 8 * k;
        int blk = p < last ? __ldg(table + p) : 0;
        const bool bad = p >= last || (unsigned)blk >= (unsigned)a.c.n_blocks;
        if (bad) {
          if (p < last && t == 0) dd_status(a.c.status, blk);
          blk = 0;
        }
        const char* lm = a.landmarks + ((long long)blk * a.c.n_kv_heads + h) * (D + CS_TAIL);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (!bad) v = *reinterpret_cast<const uint4*>(lm + t * (D / 4) + i * 16);
          r[k][4 * i] = v.x; r[k][4 * i + 1] = v.y; r[k][4 * i + 2] = v.z; r[k][4 * i + 3] = v.w;
        }
        // 2^(byte - 64), byte below 128
        by[k] = bad ? 0.f : __uint_as_float((uint32_t)((*reinterpret_cast<const unsigned char*>(lm + D) & 127) + 63) << 23);
      }
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        if (ct * 8 >= e || ct * 8 + 8 <= s) continue;
        int acc[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < D / 32; ++i) cs_mma(acc, r[0][2 * i], r[1][2 * i], r[0][2 * i + 1], r[1][2 * i + 1], qf[ct][2 * i], qf[ct][2 * i + 1]);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int i = ct * 8 + 2 * t + (x & 1), p = p0 + g + 8 * (x >> 1);
          if (i >= s && i < e) {
            const int own = sh_own[i];
            if (p <= own && p < last) {
              const bool kept = p < a.first || p > own - a.recent;
              a.keys[((long long)(n0 + i) * a.c.n_kv_heads + h) * a.stride + p] = kept ? 0xffffffffu : cs_key((float)acc[x] * by[x >> 1]);
            }
          }
        }
      }
    }
  }
}

// ---- the choice: WARPS warps per row, KPT keys a lane (0: more than fit, read again at every step). Warp w holds keys
// [w * 32 * KPT, ...), every 32nd of them a lane.
template <int WARPS, int KPT, int ROWS>
__global__ void __launch_bounds__(WARPS * ROWS * 32) dd_cache_topk_kernel(const cs_args a) {
  __shared__ int sh_n[ROWS][WARPS], sh_eq[ROWS][WARPS];
  const int lane = threadIdx.x & 31, w = (threadIdx.x >> 5) % WARPS, sub = (threadIdx.x >> 5) / WARPS;
  const long long row = (long long)blockIdx.x * ROWS + sub;
  dd_grid_dependency_wait();
  if (row >= (long long)a.n_tokens * a.c.n_kv_heads) return;         // a whole row's warps: ROWS is 1 where they share barriers
  const int n = (int)(row / a.c.n_kv_heads);
  int req;
  const int P = cs_own_page(a, a.first_token + n, req, false) + 1;
  int* out = a.out + ((long long)a.first_token * a.c.n_kv_heads + row) * a.k;
  const int k = min(a.k, P);
  for (int i = w * 32 + lane; i < a.k; i += WARPS * 32)
    if (i >= k || P <= a.k) out[i] = i < k ? i : -1;                  // everything visible fits, and what lies behind the set
  if (P <= a.k) return;
  const uint32_t* keys = a.keys + row * a.stride;
  const int span = KPT ? 32 * KPT : (P + WARPS * 32 - 1) / (WARPS * 32) * 32, at0 = w * span + lane;
  constexpr int HELD = KPT ? KPT : 1;
  uint32_t key[HELD];
  if (KPT) {
#pragma unroll
    for (int j = 0; j < HELD; ++j) key[j] = at0 + 32 * j < P ? keys[at0 + 32 * j] : 0u;      // no key is 0
  }
  auto each = [&](auto&& f) {
    if (KPT) {
#pragma unroll
      for (int j = 0; j < HELD; ++j) f(key[j], at0 + 32 * j);
    } else {
      for (int j = 0; j < span; j += 32) f(at0 + j < P ? keys[at0 + j] : 0u, at0 + j);
    }
  };
  auto total = [&](int v) {                                           // over the row
    v = __reduce_add_sync(0xffffffffu, v);
    if (WARPS == 1) return v;
    __syncthreads();
    if (lane == 0) sh_n[sub][w] = v;
    __syncthreads();
    v = lane < WARPS ? sh_n[sub][lane] : 0;
    return __reduce_add_sync(0xffffffffu, v);
  };
  // the largest x with at least k keys >= x lies in [lo, hi] (or all of these are taken along with the pages always kept)
  uint32_t lo = 0xffffffffu, hi = 0u;
  each([&](uint32_t v, int p) {
    if (p < P && v != 0xffffffffu) {
      lo = min(lo, v);
      hi = max(hi, v);
    }
  });
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (WARPS > 1) {
    if (lane == 0) { sh_n[sub][w] = (int)lo; sh_eq[sub][w] = (int)hi; }
    __syncthreads();
    lo = __reduce_min_sync(0xffffffffu, lane < WARPS ? (uint32_t)sh_n[sub][lane] : 0xffffffffu);
    hi = __reduce_max_sync(0xffffffffu, lane < WARPS ? (uint32_t)sh_eq[sub][lane] : 0u);
  }
  bool exact = false;
  // the middle of the scores at first, which splits their number better than the middle of the keys
  for (int step = 0; lo < hi; ++step) {
    uint32_t mid = lo + (hi - lo) / 2 + 1;
    if (step < 20) mid = min(max(cs_key(0.5f * cs_score(lo) + 0.5f * cs_score(hi)), lo + 1u), hi);
    int c = 0;
    each([&](uint32_t v, int) { c += v >= mid; });
    c = total(c);
    if (c == a.k) { lo = mid; exact = true; break; }
    if (c > a.k) lo = mid;
    else hi = mid - 1;
  }
  // keys >= lo where there are exactly k, else all keys > lo and the first of those that equal it
  int above = 0, equal = 0;
  each([&](uint32_t v, int) { above += v > lo; equal += v == lo; });
  above = __reduce_add_sync(0xffffffffu, above);
  equal = __reduce_add_sync(0xffffffffu, equal);
  int before = 0, before_eq = 0, all_above = above;
  if (WARPS > 1) {
    __syncthreads();
    if (lane == 0) { sh_n[sub][w] = above; sh_eq[sub][w] = equal; }
    __syncthreads();
    const int x = lane < WARPS ? sh_n[sub][lane] : 0, y = lane < WARPS ? sh_eq[sub][lane] : 0;
    all_above = __reduce_add_sync(0xffffffffu, x);
    before = __reduce_add_sync(0xffffffffu, lane < w ? x : 0);
    before_eq = __reduce_add_sync(0xffffffffu, lane < w ? y : 0);
  }
  const int take = exact ? 0x7fffffff : a.k - all_above;              // how many of the equal ones
  int at = before + min(before_eq, take), eq_at = before_eq;
  const unsigned below = (1u << lane) - 1u;
  each([&](uint32_t v, int p) {
    const unsigned eq = __ballot_sync(0xffffffffu, v == lo);
    const bool mine = v > lo || (v == lo && eq_at + __popc(eq & below) < take);
    const unsigned m = __ballot_sync(0xffffffffu, mine);
    if (mine) out[at + __popc(m & below)] = p;
    at += __popc(m);
    eq_at += __popc(eq);
  });
}

int cs_sm_count(int device) {
  int sms = 0;
  if (device < 0 || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || sms <= 0) {
    cudaGetLastError();
    return 148;
  }
  return sms;
}

template <int D> const void* cs_landmark_kernel(int format) {
  switch (format) {
    case DD_CACHE_INT4: return (const void*)dd_cache_landmark_kernel<DD_CACHE_INT4, D>;
    case DD_CACHE_E4M3: return (const void*)dd_cache_landmark_kernel<DD_CACHE_E4M3, D>;
    case DD_CACHE_FP16: return (const void*)dd_cache_landmark_kernel<DD_CACHE_FP16, D>;
    default: return (const void*)dd_cache_landmark_kernel<DD_CACHE_BF16, D>;
  }
}
template <typename T, int D> const void* cs_score_kernel(int tokens) {
  return tokens == 1 ? (const void*)dd_cache_score_kernel<T, D, 1>
                     : (tokens == 8 ? (const void*)dd_cache_score_kernel<T, D, 8> : (const void*)dd_cache_score_kernel<T, D, 64>);
}

int cs_stride(int max_pages) { return (max_pages + 31) / 32 * 32; }
// Tokens whose keys go through the workspace at a time: 64 MiB of keys stay in L2, next to the landmarks.
int cs_tokens_at_once(int n_tokens, int n_kv_heads, int max_pages) {
  const long long row = (long long)n_kv_heads * cs_stride(max_pages) * 4;
  const long long n = (64LL << 20) / row / 64 * 64;
  return (int)(n < 64 ? (n_tokens < 64 ? n_tokens : 64) : (n < n_tokens ? n : n_tokens));
}

}  // namespace

extern "C" size_t dd_cache_landmark_bytes(int head_dim) { return head_dim == 64 || head_dim == 128 ? (size_t)head_dim + CS_TAIL : 0; }

extern "C" int dd_cache_landmarks(const dd_cache* cache, const int* ctx_len, int n_last, void* landmarks, void* stream) {
  const char* who = "dd_cache_landmarks";
  DD_TRY(dd_check_cache(cache, who));
  if (n_last < 0) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: n_last is negative", who);
  const int device = dd_current_device();
  const char* data = nullptr;
  DD_TRY(dd_check_cache_memory(cache, who, device, false, &data, nullptr));
  DD_TRY(dd_check_ptr(ctx_len, who, "ctx_len", 4, device));
  DD_TRY(dd_check_ptr(landmarks, who, "landmarks", 16, device));
  dd_cache_view v = dd_make_view(cache, data);
  int pages = cache->max_pages;
  if (n_last > 0 && ((long long)n_last + cache->page_tokens - 2) / cache->page_tokens + 1 < pages)
    pages = (int)(((long long)n_last + cache->page_tokens - 2) / cache->page_tokens + 1);
  const long long warps = (long long)cache->batch * pages * cache->n_kv_heads, blocks = (warps + CL_THREADS / 32 - 1) / (CL_THREADS / 32);
  if (blocks > 0x7fffffffLL) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: too many pages", who);
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at;
  dd_pdl_attr(&at);
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(CL_THREADS);
  cfg.stream = (cudaStream_t)stream;
  void* args[] = {&v, &ctx_len, &n_last, &pages, &landmarks};
  return dd_launch(who, &cfg, cache->head_dim == 128 ? cs_landmark_kernel<128>(cache->format) : cs_landmark_kernel<64>(cache->format), args);
}

extern "C" size_t dd_cache_select_workspace(int n_tokens, int n_kv_heads, int max_pages) {
  if (n_tokens < 1 || n_kv_heads < 1 || max_pages < 1) return 0;
  return (size_t)cs_tokens_at_once(n_tokens, n_kv_heads, max_pages) * n_kv_heads * cs_stride(max_pages) * 4;
}

extern "C" int dd_cache_select(const dd_cache* cache, int n_tokens, const int* positions, const int* requests, const dd_rows* q,
                               const void* landmarks, int k_pages, int first_pages, int recent_pages, int* out_idx, void* workspace,
                               size_t workspace_bytes, void* stream) {
  const char* who = "dd_cache_select";
  DD_TRY(dd_check_cache(cache, who));
  if (n_tokens < 0) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: n_tokens is negative", who);
  if (!requests && n_tokens % cache->batch)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: without requests, n_tokens (%d) must be a multiple of batch (%d)", who, n_tokens, cache->batch);
  if (first_pages < 0 || recent_pages < 1) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: need first_pages >= 0 and recent_pages >= 1", who);
  if (k_pages < 1 || (long long)first_pages + recent_pages > k_pages)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: k_pages (%d) must hold the first %d and the last %d pages", who, k_pages, first_pages, recent_pages);
  if (n_tokens == 0) return DD_OK;
  DD_TRY(dd_check_rows(q, who, "q", cache->head_dim, n_tokens, false));
  if (q->n_heads % cache->n_kv_heads) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: n_q_heads must be a multiple of n_kv_heads", who);
  if (cache->n_kv_heads > 65535) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: too many heads", who);
  const int device = dd_current_device();
  DD_TRY(dd_check_ptr(cache->block_table, who, "cache->block_table", 4, device));
  if (cache->status) DD_TRY(dd_check_ptr(cache->status, who, "cache->status", 4, device));
  DD_TRY(dd_check_ptr(positions, who, "positions", 4, device));
  if (requests) DD_TRY(dd_check_ptr(requests, who, "requests", 4, device));
  DD_TRY(dd_check_ptr(q->data, who, "q", 16, device));
  DD_TRY(dd_check_ptr(landmarks, who, "landmarks", 16, device));
  DD_TRY(dd_check_ptr(out_idx, who, "out_idx", 4, device));
  DD_TRY(dd_check_ptr(workspace, who, "workspace", 16, device));
  const size_t need = dd_cache_select_workspace(n_tokens, cache->n_kv_heads, cache->max_pages);
  if (workspace_bytes < need) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: workspace holds %zu bytes, %zu needed", who, workspace_bytes, need);
  cs_args a = {};
  a.c = dd_make_view(cache, (const char*)cache->data);
  a.q = (const char*)q->data;
  a.q_token_stride = q->token_stride * 2;
  a.q_head_stride = q->head_stride * 2;
  a.landmarks = (const char*)landmarks;
  a.positions = positions;
  a.requests = requests;
  a.tokens_per_request = requests ? 1 : n_tokens / cache->batch;
  a.keys = (uint32_t*)workspace;
  a.out = out_idx;
  a.G = q->n_heads / cache->n_kv_heads;
  a.k = k_pages;
  a.first = first_pages;
  a.recent = recent_pages;
  a.stride = cs_stride(cache->max_pages);
  const int sms = cs_sm_count(device), each = n_tokens / cache->batch;
  // Tokens of a block: one where requests bring one or two (every token reads its own landmarks), up to 64 where they bring many.
  const int tt = each <= 2 ? 1 : (each < 32 ? 8 : 64);
  const int once = cs_tokens_at_once(n_tokens, cache->n_kv_heads, cache->max_pages);
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at;
  dd_pdl_attr(&at);
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  cfg.stream = (cudaStream_t)stream;
  void* args[] = {&a};
  for (a.first_token = 0; a.first_token < n_tokens; a.first_token += once) {
    a.n_tokens = n_tokens - a.first_token < once ? n_tokens - a.first_token : once;
    const long long tiles = (a.n_tokens + tt - 1) / tt, row_blocks = tiles * cache->n_kv_heads;
    // pages of a block: enough blocks to fill the device a few times, 64 pages at least
    const long long want = (8LL * sms + row_blocks - 1) / row_blocks;
    long long pages = ((long long)cache->max_pages + want - 1) / want;
    pages = (pages + 63) / 64 * 64;
    a.chunk_pages = (int)pages;
    a.chunks = (int)((cache->max_pages + pages - 1) / pages);
    if (tiles * a.chunks > 0x7fffffffLL) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: too many tokens", who);
    cfg.gridDim = dim3((unsigned)(tiles * a.chunks), (unsigned)cache->n_kv_heads);
    cfg.blockDim = dim3(CS_THREADS);
    const void* f = cache->head_dim == 128 ? (q->dtype == DD_BF16 ? cs_score_kernel<__nv_bfloat16, 128>(tt) : cs_score_kernel<__half, 128>(tt))
                                           : (q->dtype == DD_BF16 ? cs_score_kernel<__nv_bfloat16, 64>(tt) : cs_score_kernel<__half, 64>(tt));
    DD_TRY(dd_launch(who, &cfg, f, args));
    const long long rows = (long long)a.n_tokens * cache->n_kv_heads;
    int threads = 1024, per_block = 1;
    if (cache->max_pages <= 2048 && rows >= 4LL * sms) {
      f = (const void*)dd_cache_topk_kernel<1, 64, 4>;
      threads = 128;
      per_block = 4;
    } else if (cache->max_pages <= 4096) {
      f = (const void*)dd_cache_topk_kernel<8, 16, 1>;
      threads = 256;
    } else if (cache->max_pages <= 16384) {
      f = (const void*)dd_cache_topk_kernel<32, 16, 1>;
    } else if (cache->max_pages <= 49152) {
      f = (const void*)dd_cache_topk_kernel<32, 48, 1>;
    } else {
      f = (const void*)dd_cache_topk_kernel<32, 0, 1>;
    }
    if ((rows + per_block - 1) / per_block > 0x7fffffffLL) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: too many tokens", who);
    cfg.gridDim = dim3((unsigned)((rows + per_block - 1) / per_block));
    cfg.blockDim = dim3(threads);
    DD_TRY(dd_launch(who, &cfg, f, args));
  }
  return DD_OK;
}
