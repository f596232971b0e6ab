// Landmarks of a paged cache's pages, and the pages that each query token attends to.
//
// Landmark of (block, KV head): the mean of the page's keys as whole numbers l up to 127 times 2^e. Score of a page for query token n and
// KV head g: <c, l> * 2^e, c the sum of the group's query rows as whole numbers up to 127 (their power of two is the same for all pages of a row
// and left out). Sums and means are taken in 64 bits, where 16-bit values add up without a rounding for all but the wildest
// exponents; the product of whole numbers below 2^21 is exact whatever its order, and the power of two is exact in fp32. So the scores,
// and with them the chosen set, are defined to the last bit. (Adding up the group's rows orders pages as the product of the heads'
// soft-max probabilities does: what a head's soft-max divides by is the same for all pages.)
//
// Scores: 8-bit whole-number MMAs. They are kept as keys, numbers that compare as the scores do. Two ways, by the rule in dd_cache_select:
//   prompt chunks, many tokens   one kernel for scores and choice: 16 tokens of a head a block, the keys of all pages in shared memory
//   few rows, wide tables        a scoring kernel (1, 8 or 64 tokens a block) leaves the keys of a bounded number of tokens in a workspace that L2
//                                holds, a second one chooses. One token a block reads each landmark once (HBM: 144 bytes a page and head)
//
// Choice: the k-th largest of the maxima of small groups of keys bounds the k-th largest key from below, and the keys from there on, little more
// than k, are listed in shared memory. Few rows: every listed key's rank among the listed ones decides. Else one warp finds the k-th
// largest by bisection, a step counting keys at or above the middle, until exactly k are. Where too many are listed (ties, long lists)
// the bisection is over all keys. Equal keys go to the lower pages.
#include "dd_cache.cuh"

namespace {

// ---- 64-bit rows as whole numbers
__device__ __forceinline__ double cs_finite(double v) { return fabs(v) <= 1.7976931348623157e308 ? v : 0.0; }
// The smallest e in [least, 63] with every lane's |v| <= 127 * 2^e (v finite): 127 = 1.984375 * 2^6. The larger magnitudes have the larger
// upper words; the lower ones matter only where the upper one is 127's.
template <int N> __device__ __forceinline__ int cs_exponent(const double (&v)[N], int least) {
  unsigned hi = 0u;
#pragma unroll
  for (int i = 0; i < N; ++i) hi = max(hi, (unsigned)__double2hiint(v[i]) & 0x7fffffffu);
  hi = __reduce_max_sync(0xffffffffu, hi);
  const unsigned frac = hi & 0xfffffu;
  bool above = frac > 0xfc000u;
  if (frac == 0xfc000u) {
    bool lower = false;
#pragma unroll
    for (int i = 0; i < N; ++i) lower |= ((unsigned)__double2hiint(v[i]) & 0x7fffffffu) == hi && __double2loint(v[i]) != 0;
    above = __any_sync(0xffffffffu, lower);
  }
  return min(63, max((int)(hi >> 20) - 1023 - 6 + (above ? 1 : 0), least));
}
__device__ __forceinline__ double cs_two_to(int e) { return __hiloint2double((e + 1023) << 20, 0); }
__device__ __forceinline__ int cs_code(double v, double down) { return (int)fmin(fmax(rint(v * down), -127.0), 127.0); }
constexpr int CS_TAIL = 16;                            // bytes behind the codes of a landmark: the exponent + 64, then nothing
constexpr int CS_LM_LEAST = -64, CS_Q_LEAST = -120;

// ---- landmarks: a page and head at a time to a warp, D / 32 channels a lane. A warp takes `per` of them in a row (up to CL_PER): its lanes
// find the pages together, so that the chain length -> table entry -> keys is waited for once a warp. Bound: the 64-bit
// pipe (a widening to 64 bits and an addition for each key's channel; 0.62 to 0.7 instructions issued a cycle and scheduler), in flight 16 rows a warp. 8 x 2048 pages of 8 heads of
// 128: bf16 130 us (4.1 TB/s; one a warp 157), e4m3 148 (174), 4 bits 196 (217).
constexpr int CL_THREADS = 256, CL_PER = 8;            // in a row at most (32: 162 us where 8 took 141, the last warps being alone for too long)
// Blocks an SM: 16 rows of 16-bit keys of 128 take 32 registers, with four blocks 140 us; the others are the faster for a fourth (e4m3 158 -> 148 us).
constexpr int cl_blocks(int fmt, int d) { return d == 128 && (fmt == DD_CACHE_BF16 || fmt == DD_CACHE_FP16) ? 3 : 4; }
template <int FMT, int D>
__global__ void __launch_bounds__(CL_THREADS, (cl_blocks(FMT, D))) dd_cache_landmark_kernel(dd_cache_view c, const int* __restrict__ ctx_len, int n_last, int pages, int per, char* landmarks) {
  constexpr int N = D / 32;
  const int lane = threadIdx.x & 31;
  const long long item0 = ((long long)blockIdx.x * (CL_THREADS / 32) + (threadIdx.x >> 5)) * per;
  dd_grid_dependency_wait();
  int tokens = 0, block = 0, head = 0;                 // of the lane's page and head, no tokens = nothing to do
  if (lane < per) {
    const long long bp = (item0 + lane) / c.n_kv_heads, b = bp / pages;
    head = (int)(item0 + lane - bp * c.n_kv_heads);
    if (b < c.batch) {
      int len = ctx_len[b];
      const int most = c.max_pages << c.page_shift;
      if (len < 0 || len > most) {
        dd_status(c.status, len);
        len = len < 0 ? 0 : most;
      }
      const int from = n_last > 0 && n_last < len ? len - n_last : 0;
      const long long p = (from >> c.page_shift) + (bp - b * pages);
      if ((p << c.page_shift) < len) {
        block = c.table[b * c.table_stride + p];
        if ((unsigned)block < (unsigned)c.n_blocks) tokens = min(len - ((int)p << c.page_shift), 1 << c.page_shift);
        else dd_status(c.status, block);
      }
    }
  }
  const int T = 1 << c.page_shift;
  for (int item = 0; item < per; ++item) {
    const int n = __shfl_sync(0xffffffffu, tokens, item), blk = __shfl_sync(0xffffffffu, block, item), h = __shfl_sync(0xffffffffu, head, item);
    if (n == 0) continue;
    const char* page = c.data + blk * c.block_stride + h * c.head_stride;
    constexpr int CHAINS = 4;                            // sums that do not wait for each other
    double part[CHAINS][N], sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) part[0][i] = part[1][i] = part[2][i] = part[3][i] = 0.0;
    // 16 tokens at a time, all of their loads under way together, however many there are
    for (int t0 = 0; t0 < n; t0 += 16) {
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int t = min(t0 + j, n - 1);
        const bool in = t0 + j < n;                    // rows behind the last token are made zeros before they are widened
        float v[N];
        if (FMT == DD_CACHE_INT4) {
          const char* tile = page + (t >> 4) * dd_int4_tile_bytes(D);
          const int r = t & 15;
          const uint32_t w = N == 4 ? *reinterpret_cast<const unsigned short*>(tile + r * (D / 2) + lane * 2) : *reinterpret_cast<const unsigned char*>(tile + r * (D / 2) + lane);
          uint32_t s2, unused;
          dd_e4m3x4_to_half(*reinterpret_cast<const unsigned char*>(tile + dd_int4_ks_at<D>(r, lane * N / 16)), s2, unused);
          const float s = in ? dd_unpack2<__half>(s2).x : 0.f, by = !in ? 0.f : dd_two_to_byte(*reinterpret_cast<const unsigned char*>(tile + 18 * D + r));
#pragma unroll
          for (int i = 0; i < N; ++i) v[i] = (__uint_as_float((w >> (4 * i) & 15u) | 0x4b000000u) - 8388616.f) * s * by;      // 2^23 + code
        } else if (FMT == DD_CACHE_E4M3) {
          uint32_t w = N == 4 ? *reinterpret_cast<const uint32_t*>(page + t * D + lane * 4) : *reinterpret_cast<const unsigned short*>(page + t * D + lane * 2);
          if (!in) w = 0u;
          const float by = !in ? 0.f : dd_two_to_byte(*reinterpret_cast<const unsigned char*>(page + 2 * T * D + t));
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
          if (!in) w = make_uint2(0u, 0u);
          const float2 x = FMT == DD_CACHE_BF16 ? dd_unpack2<__nv_bfloat16>(w.x) : dd_unpack2<__half>(w.x);
          const float2 y = FMT == DD_CACHE_BF16 ? dd_unpack2<__nv_bfloat16>(w.y) : dd_unpack2<__half>(w.y);
          v[0] = x.x;
          v[1] = x.y;
          if (N == 4) { v[N - 2] = y.x; v[N - 1] = y.y; }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) part[j % CHAINS][i] += (double)v[i];
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = cs_finite(((part[0][i] + part[1][i]) + (part[2][i] + part[3][i])) / (double)n);
    const int e = cs_exponent(sum, CS_LM_LEAST);
    const double down = cs_two_to(-e);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) w |= (uint32_t)(cs_code(sum[i], down) & 0xff) << (8 * i);
    char* to = landmarks + ((long long)blk * c.n_kv_heads + h) * (D + CS_TAIL);
    if (N == 4) *reinterpret_cast<uint32_t*>(to + lane * 4) = w;
    else *reinterpret_cast<unsigned short*>(to + lane * 2) = (unsigned short)w;
    if (lane < CS_TAIL / 4) *reinterpret_cast<uint32_t*>(to + D + lane * 4) = lane == 0 ? (uint32_t)(e + 64) : 0u;
  }
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
  signed char* codes;                                  // [tokens of the launch][heads][D], where they are made ahead
  int* out;
  int first_token, n_tokens, tokens_per_request;       // tokens first_token .. first_token + n_tokens - 1
  int G, k, first, recent;
  int stride;                                          // keys of a row
  int chunks;                                          // blocks that share a token tile
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
// C(16x8, whole numbers) += A(16x32 bytes) * B(32x8 bytes)
__device__ __forceinline__ void cs_mma(int (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 2^(byte - 64), byte below 128
__device__ __forceinline__ float cs_power(unsigned byte) { return __uint_as_float(((byte & 127u) + 63u) << 23); }

// A token's queries of one head, added up and as whole numbers: one warp, D / 32 channels a lane.
template <typename T, int D>
__device__ __forceinline__ void cs_query(const cs_args& a, int n, int h, signed char* to) {
  constexpr int N = D / 32;
  const int lane = threadIdx.x & 31;
  const char* at = a.q + n * a.q_token_stride + (long long)h * a.G * a.q_head_stride + lane * (2 * N);
  double sum[N];
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] = 0.0;
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
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] = cs_finite(sum[e]);
  const double down = cs_two_to(-cs_exponent(sum, CS_Q_LEAST));
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) w |= (uint32_t)(cs_code(sum[e], down) & 0xff) << (8 * e);
  if (N == 4) *reinterpret_cast<uint32_t*>(to + lane * 4) = w;
  else *reinterpret_cast<unsigned short*>(to + lane * 2) = (unsigned short)w;
}
// The same for all tokens and heads of a launch, into the workspace: [token][head][D] bytes.
template <typename T, int D>
__global__ void __launch_bounds__(256) dd_cache_query_kernel(const cs_args a) {
  const long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  dd_grid_dependency_wait();
  if (item >= (long long)a.n_tokens * a.c.n_kv_heads) return;
  const int n = (int)(item / a.c.n_kv_heads), h = (int)(item - (long long)n * a.c.n_kv_heads);
  cs_query<T, D>(a, a.first_token + n, h, a.codes + item * D);
}

__device__ __forceinline__ void cs_copy16(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void cs_copied() { asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory"); }

// TT tokens of one head and up to cs_pages() pages, whose landmarks are brought into shared memory all at once (the chain table entry ->
// landmark is waited for once a block, not once for every few pages). A warp takes MT tiles of 16 tokens as the rows of its MMAs (their
// fragments stay in registers) and 8 pages at a time as the columns. Channels are dealt to the MMA's slots as they lie: lane t of a group of
// four takes the D / 4 channels from D / 4 t on, of landmarks and queries alike; landmarks of D + 16 bytes are read without bank
// conflicts.
DD_HD constexpr int cs_pages(int tokens) { return tokens == 1 ? 128 : 256; }
template <typename T, int D, int TT>
__global__ void __launch_bounds__(CS_THREADS) dd_cache_score_kernel(const cs_args a) {
  constexpr int ROWS = (TT + 15) / 16 * 16, MT = TT >= 32 ? 2 : 1, LM = D + CS_TAIL;
  constexpr int SETS = ROWS / (16 * MT), STRIDE = D + 16;               // warps of a set hold the same tokens and share the pages out
  constexpr int PAGES = cs_pages(TT);
  extern __shared__ __align__(16) unsigned char cs_smem[];              // landmarks [PAGES][LM]
  __shared__ __align__(16) signed char sh_q[TT][STRIDE];
  __shared__ int sh_own[ROWS], sh_req[ROWS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int set = warp % SETS, share = warp / SETS;
  constexpr int SHARES = CS_THREADS / 32 / SETS;
  const int tile = blockIdx.x / a.chunks, chunk = blockIdx.x - tile * a.chunks, h = blockIdx.y;
  const int n0 = tile * TT;                            // of the launch
  dd_grid_dependency_wait();
  if (threadIdx.x < ROWS) {
    int req = -1, own = -1;
    if (threadIdx.x < TT && n0 + threadIdx.x < a.n_tokens) own = cs_own_page(a, a.first_token + n0 + threadIdx.x, req, chunk == 0 && h == 0);
    sh_own[threadIdx.x] = own;
    sh_req[threadIdx.x] = req;
  }
  __syncthreads();
  const int p_begin = chunk * PAGES, p_end = min(p_begin + PAGES, a.c.max_pages);
  const int row0 = set * 16 * MT;
  uint32_t qf[MT][D / 32][4];                          // step s: channels D / 4 t + 8 s .. + 7 of tokens g and g + 8
  bool have_q = false;
  // tokens of one request at a time: tokens s .. e - 1 of the tile
  for (int s = 0, e; s < TT; s = e) {
    const int req = sh_req[s];
    int most = sh_own[s], least = sh_own[s];
    for (e = s + 1; e < TT && sh_req[e] == req; ++e) {
      most = max(most, sh_own[e]);
      least = min(least, sh_own[e]);
    }
    const int last = min(p_end, most + 1);
    if (p_begin >= last) continue;                     // the same for the whole block
    // ---- landmarks of pages p_begin .. last - 1
    const int* table = a.c.table + req * a.c.table_stride;
    if (s > 0) __syncthreads();                        // the pages of the tokens before have been used
    for (int i = threadIdx.x / 2; i < last - p_begin; i += CS_THREADS / 2) {       // two threads a landmark
      const int blk = __ldg(table + p_begin + i);
      unsigned char* to = cs_smem + i * LM + (threadIdx.x & 1) * 16;
      if ((unsigned)blk < (unsigned)a.c.n_blocks) {
        const char* lm = a.landmarks + ((long long)blk * a.c.n_kv_heads + h) * LM + (threadIdx.x & 1) * 16;
#pragma unroll
        for (int c = 0; c < (LM / 16 + 1) / 2; ++c)
          if (c < LM / 32 || (threadIdx.x & 1) == 0) cs_copy16(to + c * 32, lm + c * 32);
      } else {
        if (threadIdx.x % 2 == 0) dd_status(a.c.status, blk);
#pragma unroll
        for (int c = 0; c < (LM / 16 + 1) / 2; ++c)
          if (c < LM / 32 || (threadIdx.x & 1) == 0) *reinterpret_cast<uint4*>(to + c * 32) = make_uint4(0u, 0u, 0u, 0u);
      }
    }
    if (!have_q) {
      if constexpr (TT == 64) {
        for (int i = threadIdx.x; i < TT * (D / 16); i += CS_THREADS) {
          const int r = i / (D / 16), c = i % (D / 16);
          if (n0 + r < a.n_tokens) cs_copy16(&sh_q[r][c * 16], a.codes + ((long long)(n0 + r) * a.c.n_kv_heads + h) * D + c * 16);
        }
      } else {
        for (int i = warp; i < TT; i += CS_THREADS / 32)
          if (n0 + i < a.n_tokens) cs_query<T, D>(a, a.first_token + n0 + i, h, sh_q[i]);
      }
    }
    cs_copied();
    __syncthreads();
    if (!have_q) {
      have_q = true;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          const int r0 = row0 + 16 * m + g, r1 = r0 + 8;
          uint2 lo = make_uint2(0u, 0u), hi = make_uint2(0u, 0u);
          if (r0 < TT && n0 + r0 < a.n_tokens) lo = *reinterpret_cast<const uint2*>(&sh_q[r0 < TT ? r0 : 0][t * (D / 4) + 8 * i]);
          if (r1 < TT && n0 + r1 < a.n_tokens) hi = *reinterpret_cast<const uint2*>(&sh_q[r1 < TT ? r1 : 0][t * (D / 4) + 8 * i]);
          qf[m][i][0] = lo.x; qf[m][i][1] = hi.x; qf[m][i][2] = lo.y; qf[m][i][3] = hi.y;
        }
    }
    if (s >= row0 + 16 * MT || e <= row0) continue;    // none of this warp's tokens
    const bool all_rows = s <= row0 && e >= row0 + 16 * MT;
    for (int p0 = p_begin + share * 8; p0 < last; p0 += SHARES * 8) {
      // lane (g, t): D / 4 bytes of the landmark of page p0 + g (behind the last page: whatever lies there, for nobody)
      const unsigned char* lm = cs_smem + (p0 - p_begin) * LM;
      uint32_t r[D / 16];
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const uint4 v = *reinterpret_cast<const uint4*>(lm + g * LM + t * (D / 4) + i * 16);
        r[4 * i] = v.x; r[4 * i + 1] = v.y; r[4 * i + 2] = v.z; r[4 * i + 3] = v.w;
      }
      const float by0 = cs_power(lm[2 * t * LM + D]), by1 = cs_power(lm[(2 * t + 1) * LM + D]);
      int acc[MT][4];
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[m][0] = acc[m][1] = acc[m][2] = acc[m][3] = 0;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int m = 0; m < MT; ++m) cs_mma(acc[m], qf[m][i], r[2 * i], r[2 * i + 1]);
      // pages that all tokens of the run see and none of them keeps anyway
      const bool plain = all_rows && p0 >= a.first && p0 + 7 <= least - a.recent && p0 + 8 <= last;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int i = row0 + 16 * m + g + 8 * x;
          if (TT < 16 && i >= TT) continue;
          uint32_t* to = a.keys + ((long long)(n0 + i) * a.c.n_kv_heads + h) * a.stride + p0 + 2 * t;
          const uint32_t k0 = cs_key((float)acc[m][2 * x] * by0), k1 = cs_key((float)acc[m][2 * x + 1] * by1);
          if (plain) {
            *reinterpret_cast<uint2*>(to) = make_uint2(k0, k1);
          } else if (i >= s && i < e) {
            const int own = sh_own[i], page = p0 + 2 * t, end = min(own, last - 1);
            if (page <= end) to[0] = page < a.first || page > own - a.recent ? 0xffffffffu : k0;
            if (page + 1 <= end) to[1] = page + 1 < a.first || page + 1 > own - a.recent ? 0xffffffffu : k1;
          }
        }
    }
  }
}

// ---- the choice
// The k largest keys of a row that WARPS warps share; `each(f)` calls f(key, page, group) for this lane's run of pages in ascending order,
// runs in the order of the lanes, key 0 where there is no page. `count(x)` says how many of the lane's keys are x or above, and
// `list(x, f)` calls f(key, page) for those, in ascending order of their pages. The k-th largest of the maxima of small groups bounds the
// threshold from below: k keys at least are no smaller. The keys from that bound on, little more than k, are listed in shared
// memory, and one warp finds the threshold among them by bisection: a step counts keys at or above the middle, and stops as soon as
// exactly k are. Where the bound lets too many through (more than CAP; ties), the threshold is found among all keys.
template <int WARPS, int NG, int CAP, typename EACH, typename COUNT, typename LIST, typename SYNC>
__device__ __forceinline__ void cs_choose(EACH each, COUNT count, LIST list, SYNC sync, int k, int* out, int w, int* sh_a, int* sh_b, uint32_t* sh_key, unsigned* sh_page) {
  const int lane = threadIdx.x & 31;
  auto add_up = [&](int v) {                                          // over the row
    v = __reduce_add_sync(0xffffffffu, v);
    if (WARPS == 1) return v;
    sync();
    if (lane == 0) sh_a[w] = v;
    sync();
    return (int)__reduce_add_sync(0xffffffffu, lane < WARPS ? sh_a[lane] : 0);
  };
  auto range = [&](uint32_t& lo, uint32_t& hi) {
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (WARPS > 1) {
      sync();
      if (lane == 0) { sh_a[w] = (int)lo; sh_b[w] = (int)hi; }
      sync();
      lo = __reduce_min_sync(0xffffffffu, lane < WARPS ? (uint32_t)sh_a[lane] : 0xffffffffu);
      hi = __reduce_max_sync(0xffffffffu, lane < WARPS ? (uint32_t)sh_b[lane] : 0u);
    }
  };
  // The middle of two keys' scores at first, which splits their number better than the middle of the keys.
  auto middle = [&](uint32_t lo, uint32_t hi, int step) {
    return step < 20 ? min(max(cs_key(0.5f * cs_score(lo) + 0.5f * cs_score(hi)), lo + 1u), hi) : lo + (hi - lo) / 2 + 1;
  };
  // ---- the bound
  uint32_t top[NG];
#pragma unroll
  for (int i = 0; i < NG; ++i) top[i] = 0u;
  each([&](uint32_t v, int, int i) { top[i] = max(top[i], v); });
  uint32_t bound = 1u;
  {
    uint32_t lo = 0xffffffffu, hi = 0u;
#pragma unroll
    for (int i = 0; i < NG; ++i)
      if (top[i] != 0u && top[i] != 0xffffffffu) {
        lo = min(lo, top[i]);
        hi = max(hi, top[i]);
      }
    range(lo, hi);
    // at least k maxima at or above `bound` whenever it has moved; a few more than k will do
    for (int step = 0; step < 24 && lo < hi; ++step) {
      const uint32_t mid = middle(lo, hi, step);
      int c = 0;
#pragma unroll
      for (int i = 0; i < NG; ++i) c += top[i] >= mid;
      c = add_up(c);
      if (c >= k) {
        bound = lo = mid;
        if (c <= k + (k >> 3)) break;
      } else {
        hi = mid - 1;
      }
    }
  }
  // ---- the keys that are no smaller
  const int mine = count(bound);
  int before = mine;                                                  // of the lanes up to this one
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += v;
  }
  int listed = __shfl_sync(0xffffffffu, before, 31);
  before -= mine;
  if (WARPS > 1) {
    sync();
    if (lane == 0) sh_a[w] = listed;
    sync();
    const int v = lane < WARPS ? sh_a[lane] : 0;
    before += __reduce_add_sync(0xffffffffu, lane < w ? v : 0);
    listed = __reduce_add_sync(0xffffffffu, v);
  }
  if (listed <= CAP) {
    list(bound, [&](uint32_t v, int p) {
      sh_key[before] = v;
      sh_page[before] = p;
      ++before;
    });
    sync();
    if (w > 0) return;
    // one warp: entry 32 j + lane
    constexpr int FEW = 4;
    uint32_t few[FEW];
#pragma unroll
    for (int j = 0; j < FEW; ++j) few[j] = 32 * j + lane < listed ? sh_key[32 * j + lane] : 0u;
    uint32_t lo = 0xffffffffu, hi = 0u;
    auto all = [&](auto&& f) {
#pragma unroll
      for (int j = 0; j < FEW; ++j) f(few[j]);
      for (int i = 32 * FEW + lane; i < listed; i += 32) f(sh_key[i]);
    };
    all([&](uint32_t v) {
      if (v != 0u && v != 0xffffffffu) {
        lo = min(lo, v);
        hi = max(hi, v);
      }
    });
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    int take = 0x7fffffff;                                            // how many of the keys equal to the threshold
    if (listed > k) {
      bool exact = false;
      for (int step = 0; lo < hi; ++step) {
        const uint32_t mid = middle(lo, hi, step);
        int c = 0;
        all([&](uint32_t v) { c += v >= mid; });
        c = __reduce_add_sync(0xffffffffu, c);
        if (c == k) { lo = mid; exact = true; break; }
        if (c > k) lo = mid;
        else hi = mid - 1;
      }
      if (!exact) {
        int c = 0;
        all([&](uint32_t v) { c += v > lo; });
        take = k - (int)__reduce_add_sync(0xffffffffu, c);
      }
    } else {
      lo = 1u;
    }
    int at = 0, equal = 0;
    const unsigned below = (1u << lane) - 1u;
    for (int i = lane; i - lane < listed; i += 32) {
      const uint32_t v = i < listed ? sh_key[i] : 0u;
      const unsigned eq = __ballot_sync(0xffffffffu, v == lo);
      const bool in = v > lo || (v == lo && equal + __popc(eq & below) < take);
      const unsigned m = __ballot_sync(0xffffffffu, in);
      if (in) out[at + __popc(m & below)] = (int)sh_page[i];
      at += __popc(m);
      equal += __popc(eq);
    }
    return;
  }
  // ---- among all keys
  uint32_t lo = 0xffffffffu, hi = 0u;
  each([&](uint32_t v, int, int) {
    if (v != 0u && v != 0xffffffffu) {
      lo = min(lo, v);
      hi = max(hi, v);
    }
  });
  range(lo, hi);
  bool exact = false;
  for (int step = 0; lo < hi; ++step) {
    const uint32_t mid = middle(lo, hi, step);
    int c = 0;
    each([&](uint32_t v, int, int) { c += v >= mid; });
    c = add_up(c);
    if (c == k) { lo = mid; exact = true; break; }
    if (c > k) lo = mid;
    else hi = mid - 1;
  }
  int above = 0, equal = 0;
  each([&](uint32_t v, int, int) { above += v > lo; equal += v == lo; });
  int above_to = above, equal_to = equal;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, above_to, o), y = __shfl_up_sync(0xffffffffu, equal_to, o);
    if (lane >= o) {
      above_to += x;
      equal_to += y;
    }
  }
  int all_above = __shfl_sync(0xffffffffu, above_to, 31);
  const int warp_equal = __shfl_sync(0xffffffffu, equal_to, 31);
  above_to -= above;
  equal_to -= equal;
  if (WARPS > 1) {
    sync();
    if (lane == 0) { sh_a[w] = all_above; sh_b[w] = warp_equal; }
    sync();
    const int x = lane < WARPS ? sh_a[lane] : 0, y = lane < WARPS ? sh_b[lane] : 0;
    all_above = __reduce_add_sync(0xffffffffu, x);
    above_to += __reduce_add_sync(0xffffffffu, lane < w ? x : 0);
    equal_to += __reduce_add_sync(0xffffffffu, lane < w ? y : 0);
  }
  const int take = exact ? 0x7fffffff : k - all_above;
  each([&](uint32_t v, int p, int) {
    const bool eq = v == lo;
    if (v > lo || (eq && equal_to < take)) out[above_to + min(equal_to, take)] = p;
    above_to += v > lo;
    equal_to += eq;
  });
}

// Choice from keys in the workspace: WARPS warps a row, a lane's run KPT keys in registers (0: as many as it takes, read again where
// they are needed).
template <int WARPS, int KPT>
__global__ void __launch_bounds__(WARPS * 32) dd_cache_topk_kernel(const cs_args a) {
  constexpr int NG = 4, CAP = 2048;
  __shared__ int sh_a[WARPS], sh_b[WARPS];
  __shared__ uint32_t sh_key[CAP];
  __shared__ unsigned sh_page[CAP];
  const int w = threadIdx.x >> 5;
  const long long row = blockIdx.x;
  dd_grid_dependency_wait();
  const int n = (int)(row / a.c.n_kv_heads);
  int req;
  const int P = cs_own_page(a, a.first_token + n, req, false) + 1, k = a.k;
  int* out = a.out + ((long long)a.first_token * a.c.n_kv_heads + row) * k;
  if (P <= k) {                                                       // everything visible fits
    for (int i = threadIdx.x; i < k; i += WARPS * 32) out[i] = i < P ? i : -1;
    return;
  }
  const uint32_t* keys = a.keys + row * a.stride;
  const int run = KPT ? KPT : (P + WARPS * 128 - 1) / (WARPS * 128) * 4, at0 = threadIdx.x * run;
  auto load4 = [&](uint32_t* to, int at) {                            // no key is 0
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (at < P) v = *reinterpret_cast<const uint4*>(keys + at);
    to[0] = v.x;
    to[1] = at + 1 < P ? v.y : 0u;
    to[2] = at + 2 < P ? v.z : 0u;
    to[3] = at + 3 < P ? v.w : 0u;
  };
  auto choose = [&](auto each) {
    auto count = [&](uint32_t x) {
      int c = 0;
      each([&](uint32_t v, int, int) { c += v >= x; });
      return c;
    };
    auto list = [&](uint32_t x, auto&& f) {
      each([&](uint32_t v, int p, int) {
        if (v >= x) f(v, p);
      });
    };
    cs_choose<WARPS, NG, CAP>(each, count, list, [] { __syncthreads(); }, k, out, w, sh_a, sh_b, sh_key, sh_page);
  };
  if constexpr (KPT > 0) {
    uint32_t key[KPT];
#pragma unroll
    for (int j = 0; j < KPT; j += 4) load4(key + j, at0 + j);
    auto each = [&](auto&& f) {
#pragma unroll
      for (int j = 0; j < KPT; ++j) f(key[j], at0 + j, j * NG / KPT);
    };
    choose(each);
  } else {
    auto each = [&](auto&& f) {
#pragma unroll 4
      for (int j = 0; j < run; j += 4) {
        uint32_t v[4];
        load4(v, at0 + j);
#pragma unroll
        for (int i = 0; i < 4; ++i) f(v[i], at0 + j + i, i);
      }
    };
    choose(each);
  }
}

// Choice for few rows, where the chain of a bisection's steps would be what takes the time: a block of 256 threads a row, a run of up to
// 16 keys each. The k-th largest of the threads' maxima, found by every thread's rank among all (each compares its own with the 256,
// read by all at once), bounds the threshold; so does the rank of every listed key among the listed ones decide. k up to 256.
constexpr int CR_LIST = 1024, CR_RUN = 16, CR_ROW_THREADS = 256;
// Rank of entry `me` (key v) among n entries padded to a multiple of 4 with zeros: the larger keys, and of its equals those in front. The
// threads of a warp stand in a row, so that only the 32 entries around them need both questions.
__device__ __forceinline__ int cr_rank(const uint32_t* all, int n, uint32_t v, int me) {
  const uint4* all4 = reinterpret_cast<const uint4*>(all);
  const int n4 = (n + 3) >> 2, here = (me & ~31) >> 2;
  int r = 0, j = 0;
#pragma unroll 4
  for (; j < min(here, n4); ++j) {
    const uint4 o = all4[j];
    r += (o.x >= v) + (o.y >= v) + (o.z >= v) + (o.w >= v);
  }
#pragma unroll 2
  for (; j < min(here + 8, n4); ++j) {
    const uint4 o = all4[j];
    r += (o.x > v || (o.x == v && 4 * j < me)) + (o.y > v || (o.y == v && 4 * j + 1 < me)) + (o.z > v || (o.z == v && 4 * j + 2 < me)) +
         (o.w > v || (o.w == v && 4 * j + 3 < me));
  }
#pragma unroll 4
  for (; j < n4; ++j) {
    const uint4 o = all4[j];
    r += (o.x > v) + (o.y > v) + (o.z > v) + (o.w > v);
  }
  return r;
}
__global__ void __launch_bounds__(CR_ROW_THREADS) dd_cache_topk_rank_kernel(const cs_args a) {
  constexpr int WARPS = CR_ROW_THREADS / 32;
  __shared__ __align__(16) uint32_t sh_top[CR_ROW_THREADS], sh_key[CR_LIST];
  __shared__ unsigned sh_page[CR_LIST];
  __shared__ int sh_a[WARPS], sh_b[WARPS];
  __shared__ uint32_t sh_bound;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const long long row = blockIdx.x;
  dd_grid_dependency_wait();
  const int n = (int)(row / a.c.n_kv_heads);
  int req;
  const int P = cs_own_page(a, a.first_token + n, req, false) + 1, k = a.k;
  int* out = a.out + ((long long)a.first_token * a.c.n_kv_heads + row) * k;
  if (P <= k) {                                                       // everything visible fits
    for (int i = threadIdx.x; i < k; i += CR_ROW_THREADS) out[i] = i < P ? i : -1;
    return;
  }
  const uint32_t* keys = a.keys + row * a.stride;
  const int run = (P + CR_ROW_THREADS - 1) / CR_ROW_THREADS, at0 = threadIdx.x * run;
  uint32_t key[CR_RUN], top = 0u;
#pragma unroll
  for (int j = 0; j < CR_RUN; ++j) {
    key[j] = j < run && at0 + j < P ? keys[at0 + j] : 0u;             // no key is 0
    top = max(top, key[j]);
  }
  sh_top[threadIdx.x] = top;
  if (threadIdx.x == 0) sh_bound = 1u;
  __syncthreads();
  if (top != 0u && cr_rank(sh_top, CR_ROW_THREADS, top, threadIdx.x) == k - 1) sh_bound = top;
  __syncthreads();
  const uint32_t bound = sh_bound;
  auto sums = [&](int v, int& total) {                                // of the threads before this one, and of all
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) sh_a[w] = x;
    __syncthreads();
    const int y = lane < WARPS ? sh_a[lane] : 0;
    total = __reduce_add_sync(0xffffffffu, y);
    return x - v + (int)__reduce_add_sync(0xffffffffu, lane < w ? y : 0);
  };
  int mine = 0, listed;
#pragma unroll
  for (int j = 0; j < CR_RUN; ++j) mine += key[j] >= bound;
  int at = sums(mine, listed);
  if (listed <= CR_LIST) {
#pragma unroll
    for (int j = 0; j < CR_RUN; ++j)
      if (key[j] >= bound) {
        sh_key[at] = key[j];
        sh_page[at++] = at0 + j;
      }
    if (threadIdx.x < 3 && listed + threadIdx.x < CR_LIST) sh_key[listed + threadIdx.x] = 0u;
    __syncthreads();
    int done = 0;
    for (int i0 = 0; i0 < listed; i0 += CR_ROW_THREADS) {
      const int i = i0 + threadIdx.x;
      const bool in = i < listed && cr_rank(sh_key, listed, sh_key[i < listed ? i : 0], i) < k;
      int all;
      const int to = done + sums(in, all);
      if (in) out[to] = sh_page[i];
      done += all;
    }
    return;
  }
  auto each = [&](auto&& f) {
#pragma unroll
    for (int j = 0; j < CR_RUN; ++j) f(key[j], at0 + j, j / 4);
  };
  auto count = [&](uint32_t x) {
    int c = 0;
    each([&](uint32_t v, int, int) { c += v >= x; });
    return c;
  };
  auto list = [&](uint32_t x, auto&& f) {
    each([&](uint32_t v, int p, int) {
      if (v >= x) f(v, p);
    });
  };
  cs_choose<WARPS, 4, CR_LIST>(each, count, list, [] { __syncthreads(); }, k, out, w, sh_a, sh_b, sh_key, sh_page);
}

// ---- scores and choice in one, where the keys of a row fit shared memory: 16 tokens of one head against all of their pages.
// A warp brings the landmarks of 8 pages of every group of CF_PAGES, several groups ahead, multiplies them and leaves the keys in shared
// memory; then it chooses for one of the tokens. The lists of the choice lie where the landmarks were. One block an SM; what
// bounds it is latency at four warps a scheduler: the 78 M instructions of 2048 tokens x 2048 pages x 8 heads, a third of them the choice's, are 67 us
// of issue slots and take 143 us (two kernels with the keys in the workspace: 224).
constexpr int CF_PAGES = 128, CF_THREADS = 512, CF_TOKENS = 16;
constexpr int CF_STAGES = 4;
constexpr int CF_LIST = 256;                           // of a row
constexpr int CF_MOST = 2048;                          // pages
// Keys of a row in shared memory: a lane's run of pages (a multiple of 8), one word, the next lane's: no bank conflicts.
DD_HD constexpr int cf_run(int pages) { return (pages + 255) / 256 * 8; }
DD_HD constexpr int cf_stride(int max_pages) { return 32 * (cf_run(max_pages) + 1); }
size_t cf_smem(int d, int max_pages) {
  return (size_t)CF_STAGES * CF_PAGES * (d + CS_TAIL) + ((size_t)CF_TOKENS * cf_stride(max_pages) + max_pages) * 4;
}
template <typename T, int D>
__global__ void __launch_bounds__(CF_THREADS) dd_cache_select_kernel(const cs_args a) {
  constexpr int LM = D + CS_TAIL, STRIDE = D + 16, TT = CF_TOKENS, STAGES = CF_STAGES;
  static_assert(TT * CF_LIST * 8 <= STAGES * CF_PAGES * LM, "the lists lie where the landmarks were");
  static_assert(TT == CF_THREADS / 32, "a token a warp");
  extern __shared__ __align__(16) unsigned char cs_smem[];            // landmarks [STAGES][CF_PAGES][LM], keys [TT][stride], a table row
  __shared__ __align__(16) signed char sh_q[TT][STRIDE];
  __shared__ int sh_own[TT], sh_req[TT];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int h = blockIdx.y, n0 = blockIdx.x * TT, stride = cf_stride(a.c.max_pages);
  uint32_t* const keys = reinterpret_cast<uint32_t*>(cs_smem + STAGES * CF_PAGES * LM);
  int* const blocks = reinterpret_cast<int*>(keys + TT * stride);
  uint32_t* const list_key = reinterpret_cast<uint32_t*>(cs_smem);
  unsigned* const list_page = list_key + TT * CF_LIST;
  dd_grid_dependency_wait();
  if (threadIdx.x < TT) {
    int req = -1, own = -1;
    if (n0 + threadIdx.x < a.n_tokens) own = cs_own_page(a, n0 + threadIdx.x, req, h == 0);
    sh_own[threadIdx.x] = own;
    sh_req[threadIdx.x] = req;
  }
  __syncthreads();
  int furthest = 0;                                    // pages of any token of the tile
  for (int i = 0; i < TT; ++i) furthest = max(furthest, sh_own[i] + 1);
  const int run = cf_run(max(furthest, 1));
  const unsigned by_run = 0xffffffffu / run + 1;       // page / run by a multiplication (below 2^16, exact)
  uint32_t qf[D / 32][4];                              // step s: channels D / 4 t + 8 s .. + 7 of tokens g and g + 8
  bool have_q = false;
  for (int s = 0, e; s < TT; s = e) {                  // tokens of one request at a time
    const int req = sh_req[s];
    int most = sh_own[s], least = sh_own[s];
    for (e = s + 1; e < TT && sh_req[e] == req; ++e) {
      most = max(most, sh_own[e]);
      least = min(least, sh_own[e]);
    }
    if (most < a.k) continue;                          // everything they see fits (k pages and more: a choice)
    const int pages = most + 1, groups = (pages + CF_PAGES - 1) / CF_PAGES;
    const int* table = a.c.table + req * a.c.table_stride;
    const int mine = threadIdx.x >> 2, part = threadIdx.x & 3;         // four threads a landmark
    const char* const from = a.landmarks + (long long)h * LM + part * 16;
    const long long block_bytes = (long long)a.c.n_kv_heads * LM;
    unsigned char* const into = cs_smem + mine * LM + part * 16;
    auto fetch = [&](int i) {                          // group i
      const int p = i * CF_PAGES + mine;
      unsigned char* to = into + (i & (STAGES - 1)) * (CF_PAGES * LM);
      if (p < pages) {
        const int blk = blocks[p];
        if ((unsigned)blk < (unsigned)a.c.n_blocks) {
          const char* lm = from + blk * block_bytes;
#pragma unroll
          for (int c = 0; c * 64 < LM; ++c)
            if (c * 64 + 64 <= LM || part == 0) cs_copy16(to + c * 64, lm + c * 64);
        } else {
          if (part == 0) dd_status(a.c.status, blk);
#pragma unroll
          for (int c = 0; c * 64 < LM; ++c)
            if (c * 64 + 64 <= LM || part == 0) *reinterpret_cast<uint4*>(to + c * 64) = make_uint4(0u, 0u, 0u, 0u);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    __syncthreads();                                   // what the tokens before used is free
    for (int i = threadIdx.x; i < pages; i += CF_THREADS) blocks[i] = __ldg(table + i);
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < STAGES - 1; ++i) fetch(i);
    if (!have_q) {
      if (n0 + warp < a.n_tokens) cs_query<T, D>(a, n0 + warp, h, sh_q[warp]);
      __syncthreads();
      have_q = true;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        uint2 lo = make_uint2(0u, 0u), hi = make_uint2(0u, 0u);
        if (n0 + g < a.n_tokens) lo = *reinterpret_cast<const uint2*>(&sh_q[g][t * (D / 4) + 8 * i]);
        if (n0 + g + 8 < a.n_tokens) hi = *reinterpret_cast<const uint2*>(&sh_q[g + 8][t * (D / 4) + 8 * i]);
        qf[i][0] = lo.x; qf[i][1] = hi.x; qf[i][2] = lo.y; qf[i][3] = hi.y;
      }
    }
    for (int i = 0; i < groups; ++i) {
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
      __syncwarp();                                    // a warp brings the landmarks that it uses itself
      fetch(i + STAGES - 1);                           // over the group before this one
      const int p0 = i * CF_PAGES + warp * 8;
      if (p0 < pages) {
        // lane (g, t): D / 4 bytes of the landmark of page p0 + g (behind the last page: whatever lies there, for nobody)
        const unsigned char* lm = cs_smem + (i & (STAGES - 1)) * (CF_PAGES * LM) + warp * (8 * LM);
        uint32_t r[D / 16];
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
          const uint4 v = *reinterpret_cast<const uint4*>(lm + g * LM + t * (D / 4) + c * 16);
          r[4 * c] = v.x; r[4 * c + 1] = v.y; r[4 * c + 2] = v.z; r[4 * c + 3] = v.w;
        }
        const float by0 = cs_power(lm[2 * t * LM + D]), by1 = cs_power(lm[(2 * t + 1) * LM + D]);
        int acc[4] = {0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < D / 32; ++c) cs_mma(acc, qf[c], r[2 * c], r[2 * c + 1]);
        // pages that all tokens of the run see and none of them keeps anyway
        const bool plain = s == 0 && e == TT && p0 >= a.first && p0 + 7 <= least - a.recent;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int row = g + 8 * x;
          uint32_t* to = keys + row * stride + p0 + __umulhi(p0, by_run) + 2 * t;
          const uint32_t k0 = cs_key((float)acc[2 * x] * by0), k1 = cs_key((float)acc[2 * x + 1] * by1);
          if (plain) {
            to[0] = k0;
            to[1] = k1;
          } else if (row >= s && row < e) {             // (a tile of 8 pages that any token sees lies in the row whole)
            const int own = sh_own[row], page = p0 + 2 * t;
            to[0] = page > own ? 0u : (page < a.first || page > own - a.recent ? 0xffffffffu : k0);
            to[1] = page + 1 > own ? 0u : (page + 1 < a.first || page + 1 > own - a.recent ? 0xffffffffu : k1);
          }
        }
      }
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  // ---- the choice
  const int row = warp;
  if (n0 + row >= a.n_tokens) return;
  const int P = sh_own[row] + 1, k = a.k;
  int* out = a.out + ((long long)(n0 + row) * a.c.n_kv_heads + h) * k;
  if (P <= k) {                                                       // everything visible fits
    for (int i = lane; i < k; i += 32) out[i] = i < P ? i : -1;
    return;
  }
  uint32_t* const mine = keys + row * stride;
  const int at0 = lane * run;
  // zeros behind the tiles of 8 pages that were scored for this token (those of its request's furthest one here, at least its own)
  for (int p = (P + 7) / 8 * 8 + lane; p < 32 * run; p += 32) mine[p + __umulhi(p, by_run)] = 0u;
  __syncwarp();
  const uint32_t* const keys_of_lane = mine + at0 + lane;
  auto each = [&](auto&& f) {
    for (int j = 0; j < run; j += 8)
#pragma unroll
      for (int i = 0; i < 8; ++i) f(keys_of_lane[j + i], at0 + j + i, i);
  };
  auto count = [&](uint32_t x) {
    int c = 0;
    for (int j = 0; j < run; j += 8)
#pragma unroll
      for (int i = 0; i < 8; ++i) c += keys_of_lane[j + i] >= x;
    return c;
  };
  auto list = [&](uint32_t x, auto&& f) {
    for (int j = 0; j < run; j += 32) {
      unsigned bits = 0;
#pragma unroll
      for (int i8 = 0; i8 < 32; i8 += 8)
        if (j + i8 < run)
#pragma unroll
          for (int i = 0; i < 8; ++i) bits |= (keys_of_lane[j + i8 + i] >= x ? 1u : 0u) << (i8 + i);
      for (; bits; bits &= bits - 1) {
        const int i = j + __ffs(bits) - 1;
        f(keys_of_lane[i], at0 + i);
      }
    }
  };
  cs_choose<1, 8, CF_LIST>(each, count, list, [] { __syncwarp(); }, k, out, 0, nullptr, nullptr, list_key + row * CF_LIST, list_page + row * CF_LIST);
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
// Tokens whose keys go through the workspace at a time: 64 MiB of keys stay in L2, next to the landmarks; 64 tokens at least. So a launch
// has 2^24 rows and fewer blocks than 2^31.
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
  const long long items = (long long)cache->batch * pages * cache->n_kv_heads;
  int sms = 0;
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
  if (sms <= 0) sms = 148;
  // as many to a warp as leave the device full twice over
  const long long fill = items / ((long long)sms * 2 * 3 * (CL_THREADS / 32));
  int per = (int)(fill < 1 ? 1 : (fill > CL_PER ? CL_PER : fill));
  const long long warps = (items + per - 1) / per, blocks = (warps + CL_THREADS / 32 - 1) / (CL_THREADS / 32);
  if (blocks > 0x7fffffffLL) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: too many pages", who);
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at;
  dd_pdl_attr(&at);
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(CL_THREADS);
  cfg.stream = (cudaStream_t)stream;
  void* args[] = {&v, &ctx_len, &n_last, &pages, &per, &landmarks};
  return dd_launch(who, &cfg, cache->head_dim == 128 ? cs_landmark_kernel<128>(cache->format) : cs_landmark_kernel<64>(cache->format), args);
}

extern "C" size_t dd_cache_select_workspace(int n_tokens, int n_kv_heads, int max_pages) {
  if (n_tokens < 1 || n_kv_heads < 1 || n_kv_heads > 65535 || max_pages < 1 || max_pages > 0x7fffffff / 16) return 0;      // no such cache
  return (size_t)cs_tokens_at_once(n_tokens, n_kv_heads, max_pages) * n_kv_heads * (cs_stride(max_pages) * 4 + 128);
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
  const int each = n_tokens / cache->batch;
  // Tokens of a block: one where requests bring one or two (every token reads its own landmarks), up to 64 where they bring many. 8 requests
  // x 4096 pages x 8 heads, us with 1 | 8 | 64 tokens a block: 1 token each 20 | 41 | 73, 2 29 | 30 | 73, 3 41 | 35 | 78, 16 169 | 55 | 67, 31 302 | 95 | 73,
  // 64 616 | 163 | 82; one request of 31 tokens 48 | 20 | 26.
  const int tt = each <= 2 ? 1 : (each < 32 ? 8 : 64);
  const int once = cs_tokens_at_once(n_tokens, cache->n_kv_heads, cache->max_pages);
  a.codes = (signed char*)((char*)workspace + (size_t)once * cache->n_kv_heads * a.stride * 4);
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at;
  dd_pdl_attr(&at);
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  cfg.stream = (cudaStream_t)stream;
  void* args[] = {&a};
  // One kernel where requests bring more than two tokens each, a row's keys fit shared memory and there are rows enough. A tile of 16 tokens goes
  // over the pages once for each request that it touches, however few tiles there are: 2048 pages 11 us a pass and 10 for the rest, while the two
  // kernels take the longer the more rows there are. One kernel | two, us: 8 requests x 3 tokens 72 | 30, 8 x 8 32 | 23,
  // 1 x 16 22 | 13, 1 x 32 22 | 20, 1 x 40 22 | 23, 32 x 4 53 | 54, 16 x 8 32 | 38, 8 x 16 22 | 38, 1 x 2048 143 | 224; 512 pages: 1 x 32
  // (head_dim 64) 11.6 | 18.3, 96 x 3 34 | 55, 64 x 4 26 | 39; 256 pages: 1 x 16 10.6 | 12.0. One token a request, 8 of them: 22 | 14.
  const long long all_rows = (long long)n_tokens * cache->n_kv_heads, passes = (CF_TOKENS + each - 1) / (each < 1 ? 1 : each);
  int sms = 0;
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
  if (sms <= 0) sms = 148;
  if (each > 2 && cache->max_pages <= CF_MOST && all_rows * (CF_MOST / 2) >= sms * passes * cache->max_pages) {
    const bool wide = cache->head_dim == 128, bf16 = q->dtype == DD_BF16;
    const void* f = wide ? (bf16 ? (const void*)dd_cache_select_kernel<__nv_bfloat16, 128> : (const void*)dd_cache_select_kernel<__half, 128>)
                         : (bf16 ? (const void*)dd_cache_select_kernel<__nv_bfloat16, 64> : (const void*)dd_cache_select_kernel<__half, 64>);
    a.n_tokens = n_tokens;
    cfg.dynamicSmemBytes = cf_smem(cache->head_dim, cache->max_pages);
    DD_TRY(dd_allow_smem(who, f, (int)cf_smem(cache->head_dim, CF_MOST)));
    cfg.gridDim = dim3((unsigned)((n_tokens + CF_TOKENS - 1) / CF_TOKENS), (unsigned)cache->n_kv_heads);
    cfg.blockDim = dim3(CF_THREADS);
    return dd_launch(who, &cfg, f, args);
  }
  for (a.first_token = 0; a.first_token < n_tokens; a.first_token += once) {
    a.n_tokens = n_tokens - a.first_token < once ? n_tokens - a.first_token : once;
    const bool wide = cache->head_dim == 128, bf16 = q->dtype == DD_BF16;
    const void* f;
    const long long rows = (long long)a.n_tokens * cache->n_kv_heads, tiles = (a.n_tokens + tt - 1) / tt;
    const int pages = cs_pages(tt);
    a.chunks = (cache->max_pages + pages - 1) / pages;
    if (tt == 64) {
      f = wide ? (bf16 ? (const void*)dd_cache_query_kernel<__nv_bfloat16, 128> : (const void*)dd_cache_query_kernel<__half, 128>)
               : (bf16 ? (const void*)dd_cache_query_kernel<__nv_bfloat16, 64> : (const void*)dd_cache_query_kernel<__half, 64>);
      cfg.gridDim = dim3((unsigned)((rows + 7) / 8));
      cfg.blockDim = dim3(256);
      cfg.dynamicSmemBytes = 0;
      DD_TRY(dd_launch(who, &cfg, f, args));
    }
    cfg.gridDim = dim3((unsigned)(tiles * a.chunks), (unsigned)cache->n_kv_heads);
    cfg.blockDim = dim3(CS_THREADS);
    cfg.dynamicSmemBytes = (size_t)pages * (cache->head_dim + CS_TAIL);
    f = wide ? (bf16 ? cs_score_kernel<__nv_bfloat16, 128>(tt) : cs_score_kernel<__half, 128>(tt))
             : (bf16 ? cs_score_kernel<__nv_bfloat16, 64>(tt) : cs_score_kernel<__half, 64>(tt));
    if (tt == 64) DD_TRY(dd_allow_smem(who, f, (int)cfg.dynamicSmemBytes));
    DD_TRY(dd_launch(who, &cfg, f, args));
    cfg.dynamicSmemBytes = 0;
    int threads = 1024;
    if (cache->max_pages <= CR_RUN * CR_ROW_THREADS && k_pages <= CR_ROW_THREADS && rows <= 1024) {
      f = (const void*)dd_cache_topk_rank_kernel;
      threads = CR_ROW_THREADS;
    } else if (cache->max_pages <= 4096) {
      f = (const void*)dd_cache_topk_kernel<8, 16>;
      threads = 256;
    } else if (cache->max_pages <= 16384) {
      f = (const void*)dd_cache_topk_kernel<32, 16>;
    } else {
      f = (const void*)dd_cache_topk_kernel<32, 0>;
    }
    cfg.gridDim = dim3((unsigned)rows);
    cfg.blockDim = dim3(threads);
    DD_TRY(dd_launch(who, &cfg, f, args));
  }
  return DD_OK;
}
