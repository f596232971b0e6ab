// Attention of the newest tokens of every request over all of its cached tokens (paged, 16-bit or e4m3 pages).
//
// Bound: HBM. Every K and V byte of the context is read once; 4 * G flops per element and query token are far below the
// tensor peak. What has to be right is the load side: enough bytes in flight on every SM, no idle SM whatever the lengths
// are, and no pause at the border between two requests.
//
// Work split. The context of every (request, row tile, KV head) "unit" is cut into tiles of 16 tokens, and all tiles of
// the launch form one flat list, request by request. Block x of a grid that fills the device once takes an equal run of
// the list; lengths are read on the device, so the launch does not depend on them (a captured graph may be replayed with
// other lengths). The warps of a block take the tiles of its run in turn. Each warp keeps a ring of half tiles (K or V) in
// flight with 16-byte cp.async; a lane copies exactly the fragments it will use itself into its own slots of the ring, so
// no barrier, no swizzle and no bank conflict is involved, and the ring runs on across the borders of units.
//
// Arithmetic, with the up-to-8 query rows of a KV head as the N = 8 columns of the MMA (two column tiles for up to 16
// rows, several row tiles beyond):
//   S^T[token, n] = K[token, :] . q[n, :]        A = K tile, B = q^T
//   O^T[d, n]    += V^T[d, token] P^T[token, n]   A = V^T, B = P^T
// e4m3 pages: codes are exact as halves, so both products run as half MMAs on the codes. The power-of-two scale of a key
// multiplies its scores; the scale of a value is added to the exponent of its weight: with w = z + log2(scale of v) the
// running reference is the maximum of w, P = 2^(w - ref) <= 1 multiplies codes, and the denominator sums 2^(z - ref).
// The reference moves only when a weight exceeds it by 2^8 (one vote per tile instead of a reduction), so P is at most
// 2^14 after a factor 2^6 that keeps small weights out of the half's subnormals (a weight 2^-30 of the largest is still
// normal). Queries are multiplied by a power of two per row to fill the half's range: exact for every element above
// 2^-28 of the row's largest.
//
// Rounding: P to bf16 (bf16 pages; off by 2^-8 relative at most: the MMA takes both operands in one type) or half (2^-11), q
// as said, the output once. Scores, reference, denominators, accumulators and partial results are fp32.
//
// Joining. A unit inside one block is finished there. A unit cut across blocks leaves one fp32 partial per block in the
// workspace, and a second small kernel adds them in block order (always the same order: the result does not depend on
// timing); the block in which a cut unit begins writes down who takes part.
#include "dd_cache.cuh"

namespace {

constexpr int CA_WARPS = 8;
constexpr int CA_THREADS = CA_WARPS * 32;
constexpr int CA_MIN_SHARE = CA_WARPS;       // tiles per block at least: one per warp
constexpr float CA_HEADROOM = 6.f;           // log2 of the factor on P
constexpr float CA_LAZY = 8.f;               // how far (log2) a weight may exceed the reference

// formats: 0 bf16 pages and queries, 1 half pages and queries, 2 / 3 e4m3 pages with bf16 / half queries
template <int FMT> struct ca_types { using Q = __nv_bfloat16; };
template <> struct ca_types<1> { using Q = __half; };
template <> struct ca_types<3> { using Q = __half; };

template <int FMT, int D, int NT>
struct ca_geom {
  static constexpr bool FP8 = FMT >= 2;
  static constexpr int ES = FP8 ? 1 : 2;
  static constexpr int HALF_BYTES = 16 * D * ES;                      // K (or V) of a tile
  static constexpr int SLOT_BYTES = HALF_BYTES + (FP8 ? 32 : 0);      // e4m3: + exponents of the tile (in K's slot)
  static constexpr int BLOCKS_PER_SM = NT == 1 ? 2 : 1;               // two column tiles need the registers of a whole SM
  static constexpr int MERGE_BYTES = (CA_WARPS / 2) * 32 * (D / 4) * 4;
  static constexpr int RING_BUDGET = (BLOCKS_PER_SM == 2 ? 97 : 194) * 1024;
  static constexpr int STAGES_ = RING_BUDGET / (CA_WARPS * SLOT_BYTES);
  static constexpr int STAGES = STAGES_ > 12 ? 12 : STAGES_;
  static constexpr int SMEM = CA_WARPS * STAGES * SLOT_BYTES + MERGE_BYTES;
  static constexpr int NACC = D / 4;                                  // accumulator registers per column tile
  static constexpr int CH = FP8 ? 16 : 8;                             // channels per 16-byte chunk of a K row
  static constexpr int K_CHUNKS = D / (4 * CH);                       // chunks per lane and row: D/32 (16-bit), D/64 (e4m3)
};

struct ca_args {
  dd_cache_view c;
  const char* q;
  char* out;
  long long q_token_stride, q_head_stride, out_token_stride, out_head_stride;   // bytes
  const int* ctx_len;
  float* lse;
  float* part_o;       // [2 * blocks][NT][D / 4][32]
  float2* part_ml;     // [2 * blocks][NT * 8]
  int4* desc;          // [blocks]: (request, row tile * heads + head, blocks of the unit, 0) of the cut unit that begins in the block
  int n_q_heads, G, Tq, n_rows, row_tiles, window;
  float scale_log2;
};

__device__ __forceinline__ void ca_cp16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ca_cp8(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ca_cp4(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ca_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void ca_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 ca_lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 ca_lds8(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ int ca_lds_byte(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return (int)v;
}
__device__ __forceinline__ void ca_mma_half(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <int FMT>
__device__ __forceinline__ void ca_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (FMT == 0) dd_mma_bf16(c, a0, a1, a2, a3, b0, b1);
  else ca_mma_half(c, a0, a1, a2, a3, b0, b1);
}
__device__ __forceinline__ uint32_t ca_transpose(uint32_t a) {       // 8x8 matrix of 16-bit values across the warp
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ float ca_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t ca_word(const uint4& v, int w) { return w == 0 ? v.x : (w == 1 ? v.y : (w == 2 ? v.z : v.w)); }

// Tokens [first, end) of a request that any of its query tokens sees, as tiles of 16.
struct ca_span {
  int end, first;      // tokens; first is the lowest visible one
  int tile0, tiles;
};
__device__ __forceinline__ ca_span ca_span_of(const ca_args& a, int b, bool report) {
  int len = a.ctx_len[b];
  const int most = a.c.max_pages << a.c.page_shift;
  if (len < 0 || len > most) {
    if (report) dd_status(a.c.status, len);
    len = len < 0 ? 0 : most;
  }
  ca_span s;
  s.end = len;
  s.first = 0;
  if (a.window > 0) {
    const long long f = (long long)len - a.Tq - a.window + 1;
    s.first = f > 0 ? (int)f : 0;
  }
  s.tile0 = s.first >> 4;
  s.tiles = len > 0 ? ((len + 15) >> 4) - s.tile0 : 0;
  return s;
}

// A place in the flat list of tiles.
struct ca_cursor {
  int b, sub, t;       // request, row tile * heads + head, tile of the unit
  ca_span s;
};
__device__ __forceinline__ void ca_advance(const ca_args& a, ca_cursor& k, int by, int subs) {
  k.t += by;
  while (k.t >= k.s.tiles) {
    k.t -= k.s.tiles;
    if (++k.sub == subs) {
      k.sub = 0;
      do {
        if (++k.b >= a.c.batch) { k.b = a.c.batch - 1; k.s.tiles = 0x7fffffff; return; }   // behind the last tile: never used
        k.s = ca_span_of(a, k.b, false);
      } while (k.s.tiles == 0);
    }
  }
}

__device__ __forceinline__ int ca_channel(bool fp8, int D, int g, int m) {      // channel of accumulator row g of V product m
  return fp8 ? (D / 8) * g + 2 * m : (m >> 2) * 64 + 8 * g + 2 * (m & 3);
}

template <int FMT, int D, int NT>
__global__ void __launch_bounds__(CA_THREADS, (ca_geom<FMT, D, NT>::BLOCKS_PER_SM)) dd_cache_attn_kernel(const ca_args a) {
  using geo = ca_geom<FMT, D, NT>;
  using TQ = typename ca_types<FMT>::Q;
  constexpr bool FP8 = geo::FP8;
  constexpr int NS = geo::STAGES;
  extern __shared__ __align__(16) unsigned char ca_smem[];
  __shared__ long long sh_scan[CA_WARPS];
  __shared__ int sh_start[3];
  __shared__ float2 sh_ml[CA_WARPS][NT * 8];

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  const int subs = a.row_tiles * a.c.n_kv_heads;
  const int B = a.c.batch;

  dd_grid_dependency_wait();

  // ---- this block's run of the flat list
  long long mine = 0;
  const int chunk = (B + CA_THREADS - 1) / CA_THREADS;
  const int b_lo = min(B, (int)threadIdx.x * chunk), b_hi = min(B, b_lo + chunk);
  for (int b = b_lo; b < b_hi; ++b) mine += (long long)ca_span_of(a, b, blockIdx.x == 0).tiles * subs;
  long long incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) sh_scan[warp] = incl;
  __syncthreads();
  long long total = 0, before = 0;
#pragma unroll
  for (int w = 0; w < CA_WARPS; ++w) {
    if (w < warp) before += sh_scan[w];
    total += sh_scan[w];
  }
  long long share = (total + gridDim.x - 1) / gridDim.x;
  if (share < CA_MIN_SHARE) share = CA_MIN_SHARE;
  const long long f0 = share * blockIdx.x;
  const long long f1 = f0 + share < total ? f0 + share : total;
  {
    long long at = before + incl - mine;             // first tile of this thread's requests
    if (f0 < total && f0 >= at && f0 < at + mine) {
      for (int b = b_lo; b < b_hi; ++b) {
        const int nt = ca_span_of(a, b, false).tiles;
        const long long n = (long long)nt * subs;
        if (f0 < at + n) {
          sh_start[0] = b;
          sh_start[1] = (int)((f0 - at) / nt);
          sh_start[2] = (int)((f0 - at) % nt);
          break;
        }
        at += n;
      }
    }
  }
  __syncthreads();

  // ---- units without a token: zeros and -inf, shared out over the blocks
  for (int b = blockIdx.x; b < B; b += gridDim.x) {
    if (ca_span_of(a, b, false).tiles == 0) {
      for (int i = threadIdx.x; i < a.Tq * a.n_q_heads * (D / 8); i += CA_THREADS) {
        const int row = i / (D / 8), tok = row / a.n_q_heads, h = row - tok * a.n_q_heads;
        char* o = a.out + ((long long)b * a.Tq + tok) * a.out_token_stride + h * a.out_head_stride;
        *reinterpret_cast<uint4*>(o + (i % (D / 8)) * 16) = make_uint4(0u, 0u, 0u, 0u);
        if (a.lse && i % (D / 8) == 0) a.lse[((long long)b * a.Tq + tok) * a.n_q_heads + h] = -INFINITY;
      }
    }
  }
  if (f0 >= total) {
    if (threadIdx.x == 0) a.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
    return;
  }

  // ---- the issuing side: this warp's tiles are f0 + warp, + CA_WARPS, ...
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ca_smem) + warp * NS * geo::SLOT_BYTES;
  float* merge = reinterpret_cast<float*>(ca_smem + CA_WARPS * NS * geo::SLOT_BYTES);
  const int span = (int)(f1 - f0);
  int left = span > warp ? (span - warp - 1) / CA_WARPS + 1 : 0;      // tiles not yet issued
  ca_cursor is;
  is.b = sh_start[0]; is.sub = sh_start[1]; is.t = sh_start[2];
  is.s = ca_span_of(a, is.b, false);
  if (left > 0) ca_advance(a, is, warp, subs);
  const int page_mask = (1 << a.c.page_shift) - 1;

  auto block_of = [&](const ca_cursor& k) {          // table entry of a tile, -1 if it names no block
    const int blk = __ldg(a.c.table + k.b * a.c.table_stride + (((k.s.tile0 + k.t) << 4) >> a.c.page_shift));
    return blk;
  };
  int next_blk = left > 0 ? block_of(is) : 0;
  const char* src = nullptr;                         // K of the tile being issued; V lies page_tokens rows behind
  int n_first = 0, n_valid = 0;                      // tokens [n_first, n_valid) of it exist (and are visible to some row)
  bool second = false;                               // the next half to issue is V
  int put = 0;                                       // slot it goes to

  auto issue = [&]() {
    if (left > 0) {
      const uint32_t dst = ring + put * geo::SLOT_BYTES;
      if (!second) {
        const int tok0 = (is.s.tile0 + is.t) << 4;
        const int head = is.sub % a.c.n_kv_heads;
        int blk = next_blk;
        n_first = is.s.first - tok0;
        n_valid = is.s.end - tok0;
        if ((unsigned)blk >= (unsigned)a.c.n_blocks) {
          if (lane == 0) dd_status(a.c.status, blk);
          blk = 0;
          n_valid = 0;                               // reads as zeros
        }
        src = a.c.data + blk * a.c.block_stride + head * a.c.head_stride + (long long)(tok0 & page_mask) * (D * geo::ES);
        const uint32_t ok0 = (g >= n_first && g < n_valid) ? 16u : 0u, ok1 = (g + 8 >= n_first && g + 8 < n_valid) ? 16u : 0u;
#pragma unroll
        for (int s = 0; s < geo::K_CHUNKS; ++s) {
          const char* p = src + g * (D * geo::ES) + (t + 4 * s) * 16;
          ca_cp16(dst + (2 * s) * 512 + lane * 16, p, ok0);
          ca_cp16(dst + (2 * s + 1) * 512 + lane * 16, p + 8 * D * geo::ES, ok1);
        }
        if (FP8 && lane < 8) {
          // exponents: K's behind all the codes of the page, V's behind those
          const int in_page = tok0 & page_mask;
          const char* ex = src - in_page * D + (2 * D + (lane >= 4 ? 1 : 0)) * (page_mask + 1) + in_page + (lane & 3) * 4;
          ca_cp4(dst + geo::HALF_BYTES + lane * 4, ex, n_valid > 0 ? 4u : 0u);
        }
        second = true;
      } else {
        const char* vp = src + (long long)(page_mask + 1) * (D * geo::ES);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int tok = 2 * t + (k & 1) + (k >> 1) * 8;
          const bool ok = tok >= n_first && tok < n_valid;
          if (FP8 && D == 64) {
            ca_cp8(dst + k * 256 + lane * 8, vp + tok * D + g * 8, ok ? 8u : 0u);
          } else if (FP8) {
            ca_cp16(dst + k * 512 + lane * 16, vp + tok * D + g * 16, ok ? 16u : 0u);
          } else {
#pragma unroll
            for (int c = 0; c < D / 64; ++c)
              ca_cp16(dst + (k * (D / 64) + c) * 512 + lane * 16, vp + tok * (2 * D) + c * 128 + g * 16, ok ? 16u : 0u);
          }
        }
        second = false;
        if (--left > 0) {
          ca_advance(a, is, CA_WARPS, subs);
          next_blk = block_of(is);
        }
      }
    }
    ca_commit();
    put = put + 1 == NS ? 0 : put + 1;
  };
#pragma unroll 1
  for (int i = 0; i < NS; ++i) issue();
  int take = 0;                                      // slot of the next half to use

  // ---- the using side, unit by unit
  int b = sh_start[0], sub = sh_start[1], t0 = sh_start[2];
  ca_span s = ca_span_of(a, b, false);
  int4 desc = make_int4(0, 0, 0, 0);
  for (long long f = f0; f < f1;) {
    const int n_here = (int)min((long long)(s.tiles - t0), f1 - f);   // tiles of the unit in this block
    if (n_here <= 0) break;                                           // lengths changed under the call: stop
    const int rt = sub / a.c.n_kv_heads, head = sub - rt * a.c.n_kv_heads;
    const int r0 = rt * NT * 8;                                       // first row of the tile

    // query fragments: column n = g of column tile nt is row r0 + 8 nt + g
    uint32_t qf[NT][D / 8];
    float zs[NT][2];
    int pos[NT][2];                                                   // position of the lane's two columns, -1 = no such row
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = r0 + nt * 8 + g;
      uint2 w[D / 16];
      if (row < a.n_rows) {
        const int tok = row / a.G;
        const char* qr = a.q + ((long long)b * a.Tq + tok) * a.q_token_stride + (head * a.G + row - tok * a.G) * a.q_head_stride;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const int ch = (t + 4 * (ks / (geo::CH / 4))) * geo::CH + 4 * (ks % (geo::CH / 4));
          w[ks] = *reinterpret_cast<const uint2*>(qr + 2 * ch);
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) w[ks] = make_uint2(0u, 0u);
      }
      float back = 1.f;                                               // what the row was divided by
      if (FP8) {
        float amax = 0.f;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const float2 u0 = dd_unpack2<TQ>(w[ks].x), u1 = dd_unpack2<TQ>(w[ks].y);
          amax = fmaxf(amax, fmaxf(fmaxf(fabsf(u0.x), fabsf(u0.y)), fmaxf(fabsf(u1.x), fabsf(u1.y))));
        }
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        // the largest element lands in [2^14, 2^15); zero and non-finite rows stay as they are
        int e = (int)(__float_as_uint(amax) >> 23) - 127 - 14;
        if (!(amax > 0.f) || !(amax <= 3.4028234e38f)) e = 0;
        e = max(e, -126);
        const float by = __uint_as_float((uint32_t)(127 - e) << 23);
        back = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const float2 u0 = dd_unpack2<TQ>(w[ks].x), u1 = dd_unpack2<TQ>(w[ks].y);
          w[ks].x = dd_pack2<__half>(u0.x * by, u0.y * by);
          w[ks].y = dd_pack2<__half>(u1.x * by, u1.y * by);
        }
      }
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) { qf[nt][2 * ks] = w[ks].x; qf[nt][2 * ks + 1] = w[ks].y; }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        zs[nt][c] = a.scale_log2 * (FP8 ? __shfl_sync(0xffffffffu, back, (2 * t + c) * 4) : 1.f);
        const int r = r0 + nt * 8 + 2 * t + c;
        pos[nt][c] = r < a.n_rows ? s.end - a.Tq + r / a.G : -1;
      }
    }
    const int pos_lo = s.end - a.Tq + r0 / a.G;                       // positions of the first and last row of the tile
    const int pos_hi = s.end - a.Tq + (min(a.n_rows, r0 + NT * 8) - 1) / a.G;

    float acc[NT][D / 16][4];
    float ref[NT][2], sum[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int m = 0; m < D / 16; ++m) acc[nt][m][0] = acc[nt][m][1] = acc[nt][m][2] = acc[nt][m][3] = 0.f;
      ref[nt][0] = ref[nt][1] = -INFINITY;
      sum[nt][0] = sum[nt][1] = 0.f;
    }

    int i = (warp - (int)((f - f0) % CA_WARPS) + CA_WARPS) % CA_WARPS;   // first tile of the segment that is this warp's
    for (; i < n_here; i += CA_WARPS) {
      const int tok0 = (s.tile0 + t0 + i) << 4;
      // ---- scores
      float z[NT][4];
      int kex0 = 0, kex1 = 0, vex0 = 0, vex1 = 0;
      ca_wait<NS - 1>();
      if (FP8) __syncwarp();
      {
        const uint32_t slot = ring + take * geo::SLOT_BYTES;
        float z2[NT][4];                                              // two chains: the products of one depend on each other
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          z[nt][0] = z[nt][1] = z[nt][2] = z[nt][3] = z2[nt][0] = z2[nt][1] = z2[nt][2] = z2[nt][3] = 0.f;
#pragma unroll
        for (int c = 0; c < geo::K_CHUNKS; ++c) {
          const uint4 lo = ca_lds16(slot + (2 * c) * 512 + lane * 16), hi = ca_lds16(slot + (2 * c + 1) * 512 + lane * 16);
          if (FP8) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              uint32_t a0, a1, a2, a3;
              dd_e4m3x4_to_half(ca_word(lo, w), a0, a2);
              dd_e4m3x4_to_half(ca_word(hi, w), a1, a3);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
                ca_mma<FMT>((w & 1) ? z2[nt] : z[nt], a0, a1, a2, a3, qf[nt][2 * (4 * c + w)], qf[nt][2 * (4 * c + w) + 1]);
            }
          } else {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              ca_mma<FMT>(z[nt], lo.x, hi.x, lo.y, hi.y, qf[nt][4 * c], qf[nt][4 * c + 1]);
              ca_mma<FMT>(z2[nt], lo.z, hi.z, lo.w, hi.w, qf[nt][4 * c + 2], qf[nt][4 * c + 3]);
            }
          }
        }
        if (FP8) {
          kex0 = ca_lds_byte(slot + geo::HALF_BYTES + g);
          kex1 = ca_lds_byte(slot + geo::HALF_BYTES + g + 8);
          vex0 = ca_lds_byte(slot + geo::HALF_BYTES + 16 + g) - 127;
          vex1 = ca_lds_byte(slot + geo::HALF_BYTES + 16 + g + 8) - 127;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            z[nt][e] = (z[nt][e] + z2[nt][e]) * zs[nt][e & 1];
            if (FP8) z[nt][e] *= dd_two_to_byte(e < 2 ? kex0 : kex1);
          }
      }
      if (FP8) __syncwarp();                                          // the exponents have been read: the slot may be refilled
      take = take + 1 == NS ? 0 : take + 1;
      issue();

      // ---- masks: z[.][0..1] is token tok0 + g, z[.][2..3] token tok0 + g + 8
      const bool partial = tok0 + 15 > pos_lo || (a.window > 0 && tok0 <= pos_hi - a.window);
      if (partial) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int tok = tok0 + g + (e < 2 ? 0 : 8), p = pos[nt][e & 1];
            if (tok > p || (a.window > 0 && tok <= p - a.window)) z[nt][e] = -INFINITY;
          }
      }

      // ---- weights against the reference
      uint32_t pb[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = FP8 ? z[nt][e] + (float)max(e < 2 ? vex0 : vex1, -96) : z[nt][e];
        const bool above = w[0] > ref[nt][0] + CA_LAZY || w[2] > ref[nt][0] + CA_LAZY ||
                           w[1] > ref[nt][1] + CA_LAZY || w[3] > ref[nt][1] + CA_LAZY;
        if (__any_sync(0xffffffffu, above)) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float top = fmaxf(w[c], w[2 + c]);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
            top = fmaxf(top, ref[nt][c]);
            const float fix = top == -INFINITY ? 1.f : ca_exp2(ref[nt][c] - top);
            ref[nt][c] = top;
            sum[nt][c] *= fix;
#pragma unroll
            for (int m = 0; m < D / 16; ++m) { acc[nt][m][c] *= fix; acc[nt][m][2 + c] *= fix; }
          }
        }
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float from = (ref[nt][e & 1] == -INFINITY ? 0.f : ref[nt][e & 1]) - CA_HEADROOM;
          if (FP8) {
            const int ve = e < 2 ? vex0 : vex1;
            sum[nt][e & 1] += ca_exp2(z[nt][e] - from);
            p[e] = ca_exp2(z[nt][e] + (float)ve - from);
          } else {
            p[e] = ca_exp2(z[nt][e] - from);
            sum[nt][e & 1] += p[e];
          }
        }
        using TP = typename ca_types<FMT == 0 ? 0 : 1>::Q;
        pb[nt][0] = ca_transpose(dd_pack2<TP>(p[0], p[1]));
        pb[nt][1] = ca_transpose(dd_pack2<TP>(p[2], p[3]));
      }

      // ---- weighted values
      ca_wait<NS - 1>();
      {
        const uint32_t slot = ring + take * geo::SLOT_BYTES;
        // Tokens seen by some rows of the tile and not by others: a weight of zero does not keep an infinity or NaN of V
        // out of the sum, so the products are taken query token by query token with the unseen values replaced by zeros.
        const bool mixed = partial && a.Tq > 1;
        for (int p = mixed ? pos_lo : pos_hi; p <= pos_hi; ++p) {
          uint4 v[4][(D + 63) / 64];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (FP8 && D == 64) {
              const uint2 h = ca_lds8(slot + k * 256 + lane * 8);
              v[k][0] = make_uint4(h.x, h.y, 0u, 0u);
            } else if (FP8) {
              v[k][0] = ca_lds16(slot + k * 512 + lane * 16);
            } else {
#pragma unroll
              for (int c = 0; c < D / 64; ++c) v[k][c] = ca_lds16(slot + (k * (D / 64) + c) * 512 + lane * 16);
            }
            if (mixed) {
              const int tok = tok0 + 2 * t + (k & 1) + (k >> 1) * 8;
              if (tok > p || (a.window > 0 && tok <= p - a.window)) {
#pragma unroll
                for (int c = 0; c < (D + 63) / 64; ++c) v[k][c] = make_uint4(0u, 0u, 0u, 0u);
              }
            }
          }
#pragma unroll
          for (int m = 0; m < D / 16; ++m) {
            uint32_t a0, a1, a2, a3;
            if (FP8) {
              // bytes 2(m&1), 2(m&1)+1 of word m / 2: two channels; tokens 2t | 2t+1 side by side, then as halves
              const uint32_t sel = (m & 1) ? 0x7362u : 0x5140u;
              dd_e4m3x4_to_half(__byte_perm(ca_word(v[0][0], m >> 1), ca_word(v[1][0], m >> 1), sel), a0, a1);
              dd_e4m3x4_to_half(__byte_perm(ca_word(v[2][0], m >> 1), ca_word(v[3][0], m >> 1), sel), a2, a3);
            } else {
              const int c = m >> 2, w = m & 3;
              a0 = __byte_perm(ca_word(v[0][c], w), ca_word(v[1][c], w), 0x5410u);
              a1 = __byte_perm(ca_word(v[0][c], w), ca_word(v[1][c], w), 0x7632u);
              a2 = __byte_perm(ca_word(v[2][c], w), ca_word(v[3][c], w), 0x5410u);
              a3 = __byte_perm(ca_word(v[2][c], w), ca_word(v[3][c], w), 0x7632u);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              if (!mixed) {
                ca_mma<FMT>(acc[nt][m], a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
              } else {
                float one[4] = {0.f, 0.f, 0.f, 0.f};
                ca_mma<FMT>(one, a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (pos[nt][e & 1] == p) acc[nt][m][e] += one[e];
              }
            }
          }
        }
      }
      take = take + 1 == NS ? 0 : take + 1;
      issue();
    }

    // ---- the block's result for the unit: warps merged pairwise, always in the same order
    const bool whole = t0 == 0 && n_here == s.tiles;
    const int slot_of_block = 2 * blockIdx.x + (t0 == 0 ? 1 : 0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        sum[nt][c] += __shfl_xor_sync(0xffffffffu, sum[nt][c], 4);
        sum[nt][c] += __shfl_xor_sync(0xffffffffu, sum[nt][c], 8);
        sum[nt][c] += __shfl_xor_sync(0xffffffffu, sum[nt][c], 16);
        if (g == 0) sh_ml[warp][nt * 8 + 2 * t + c] = make_float2(ref[nt][c], sum[nt][c]);
      }
    __syncthreads();
    float top[NT][2], den[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < CA_WARPS; ++w) M = fmaxf(M, sh_ml[w][nt * 8 + 2 * t + c].x);
#pragma unroll
        for (int w = 0; w < CA_WARPS; ++w) {
          const float2 ml = sh_ml[w][nt * 8 + 2 * t + c];
          L += ml.x == -INFINITY ? ml.y : ml.y * ca_exp2(ml.x - M);   // a warp without a finite weight still passes on a NaN
        }
        top[nt][c] = M;
        den[nt][c] = L;
        const float fix = ref[nt][c] == -INFINITY ? 1.f : ca_exp2(ref[nt][c] - M);
#pragma unroll
        for (int m = 0; m < D / 16; ++m) { acc[nt][m][c] *= fix; acc[nt][m][2 + c] *= fix; }
      }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int half = CA_WARPS / 2; half >= 1; half >>= 1) {
        if (warp >= half && warp < 2 * half) {
#pragma unroll
          for (int m = 0; m < D / 16; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) merge[((warp - half) * geo::NACC + m * 4 + e) * 32 + lane] = acc[nt][m][e];
        }
        __syncthreads();
        if (warp < half) {
#pragma unroll
          for (int m = 0; m < D / 16; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[nt][m][e] += merge[(warp * geo::NACC + m * 4 + e) * 32 + lane];
        }
        __syncthreads();
      }
    }
    if (warp == 0) {
      if (whole) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int r = r0 + nt * 8 + 2 * t + c;
            if (r < a.n_rows) {
              const int tok = r / a.G, h = head * a.G + r - tok * a.G;
              const long long tn = (long long)b * a.Tq + tok;
              const bool empty = pos[nt][c] < 0;
              const float inv = empty ? 0.f : 1.f / den[nt][c];
              char* o = a.out + tn * a.out_token_stride + h * a.out_head_stride;
#pragma unroll
              for (int k = 0; k < D / 64; ++k) {
                uint32_t w[4];
#pragma unroll
                for (int q = 0; q < 4; ++q)
                  w[q] = empty ? 0u : dd_pack2<TQ>(acc[nt][4 * k + q][c] * inv, acc[nt][4 * k + q][2 + c] * inv);
                *reinterpret_cast<uint4*>(o + 2 * ca_channel(FP8, D, g, 4 * k)) = make_uint4(w[0], w[1], w[2], w[3]);
              }
              if (a.lse && g == 0)
                a.lse[tn * a.n_q_heads + h] = empty ? -INFINITY : (top[nt][c] - CA_HEADROOM + log2f(den[nt][c])) * 0.6931471805599453f;
            }
          }
      } else {
        float* po = a.part_o + (long long)slot_of_block * NT * geo::NACC * 32;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int m = 0; m < D / 16; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) po[(nt * geo::NACC + m * 4 + e) * 32 + lane] = acc[nt][m][e];
          if (g == 0) {
            a.part_ml[(long long)slot_of_block * NT * 8 + nt * 8 + 2 * t] = make_float2(top[nt][0], den[nt][0]);
            a.part_ml[(long long)slot_of_block * NT * 8 + nt * 8 + 2 * t + 1] = make_float2(top[nt][1], den[nt][1]);
          }
        }
      }
    }
    if (t0 == 0 && !whole)                                            // the last unit of the run, going on in the next blocks
      desc = make_int4(b, sub, (int)((f + s.tiles - 1) / share - blockIdx.x) + 1, 0);

    // ---- the next unit
    f += n_here;
    t0 = 0;
    if (f < f1) {
      if (++sub == subs) {
        sub = 0;
        do { s = ca_span_of(a, ++b, false); } while (s.tiles == 0 && b < B - 1);
      }
    }
  }
  ca_wait<0>();
  if (threadIdx.x == 0) a.desc[blockIdx.x] = desc;
}

// Adds the partials of the unit that begins in block x of the attention kernel and goes on in the following ones.
// Grid (blocks of the attention kernel, NT * D / 32): every thread owns one accumulator element.
template <int FMT, int D, int NT>
__global__ void __launch_bounds__(256) dd_cache_attn_join_kernel(const ca_args a, int max_parts) {
  using TQ = typename ca_types<FMT>::Q;
  constexpr int NACC = D / 4;
  extern __shared__ float ja_scale[];                                 // [parts][8] of the column tile
  __shared__ float2 sh_ml[8];
  dd_grid_dependency_wait();
  const int4 d = a.desc[blockIdx.x];
  const int n = min(d.z, max_parts);
  if (n == 0) return;
  const int e = blockIdx.y * 256 + threadIdx.x;                       // element: [nt][register][lane]
  const int nt = (blockIdx.y * 256) / (NACC * 32);
  const long long first = 2LL * blockIdx.x + 1;                       // the unit's own block leaves its partial in its second slot
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto slot = [&](int i) { return i == 0 ? first : 2LL * (blockIdx.x + i); };
  {
    // warp w: the scales of row w of the column tile
    const int row = nt * 8 + warp;
    float M = -INFINITY;
    for (int i = lane; i < n; i += 32) M = fmaxf(M, a.part_ml[slot(i) * NT * 8 + row].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    float L = 0.f;
    for (int i = lane; i < n; i += 32) {
      const float2 ml = a.part_ml[slot(i) * NT * 8 + row];
      const float sc = ml.x == -INFINITY ? 1.f : ca_exp2(ml.x - M);   // nothing but zeros (or NaN) there
      ja_scale[i * 8 + warp] = sc;
      L += ml.y * sc;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
    if (lane == 0) sh_ml[warp] = make_float2(M, L);
  }
  __syncthreads();
  const int reg = (e / 32) % NACC, m = reg >> 2, g = lane >> 2, t = lane & 3;
  const int col = 2 * t + (reg & 1);
  float acc = 0.f;
#pragma unroll 8
  for (int i = 0; i < n; ++i) acc = fmaf(a.part_o[slot(i) * (NT * NACC * 32) + e], ja_scale[i * 8 + col], acc);
  const int rt = d.y / a.c.n_kv_heads, head = d.y - rt * a.c.n_kv_heads;
  const int r = rt * NT * 8 + nt * 8 + col;
  if (r >= a.n_rows) return;
  const ca_span s = ca_span_of(a, d.x, false);
  const int tok = r / a.G, h = head * a.G + r - tok * a.G;
  const long long tn = (long long)d.x * a.Tq + tok;
  const bool empty = s.end - a.Tq + tok < 0;
  const float2 ml = sh_ml[col];
  const int ch = ca_channel(FMT >= 2, D, g, m) + ((reg >> 1) & 1);
  TQ* o = reinterpret_cast<TQ*>(a.out + tn * a.out_token_stride + h * a.out_head_stride);
  const uint32_t w = dd_pack2<TQ>(empty ? 0.f : acc / ml.y, 0.f);
  o[ch] = *reinterpret_cast<const TQ*>(&w);
  if (a.lse && ch == 0) a.lse[tn * a.n_q_heads + h] = empty ? -INFINITY : (ml.x - CA_HEADROOM + log2f(ml.y)) * 0.6931471805599453f;
}

struct ca_plan {
  const void* main_kernel;
  const void* join_kernel;
  int smem, blocks_per_sm, nt;
};
template <int FMT, int D, int NT> ca_plan ca_plan_of() {
  using geo = ca_geom<FMT, D, NT>;
  static_assert(geo::SMEM <= 227 * 1024, "shared memory of a block");
  static_assert(geo::BLOCKS_PER_SM == 1 || geo::SMEM + 2048 <= 114 * 1024, "shared memory of two blocks");
  return {(const void*)dd_cache_attn_kernel<FMT, D, NT>, (const void*)dd_cache_attn_join_kernel<FMT, D, NT>, geo::SMEM, geo::BLOCKS_PER_SM, NT};
}
template <int FMT> ca_plan ca_pick(int d, int nt) {
  if (d == 128) return nt == 1 ? ca_plan_of<FMT, 128, 1>() : ca_plan_of<FMT, 128, 2>();
  return nt == 1 ? ca_plan_of<FMT, 64, 1>() : ca_plan_of<FMT, 64, 2>();
}

int ca_sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms <= 0) {
    cudaGetLastError();
    return 148;
  }
  return sms;
}

// Rows of a unit that go through the MMA together: up to 8 in one column tile, up to 16 in two.
int ca_column_tiles(int rows) { return rows <= 8 ? 1 : 2; }

struct ca_sizes { size_t part_o, part_ml, desc; size_t total() const { return part_o + part_ml + desc; } };
ca_sizes ca_size(int head_dim, int rows, int sms) {
  const int nt = ca_column_tiles(rows);
  const size_t blocks = (size_t)sms * (nt == 1 ? 2 : 1);
  ca_sizes z;
  z.part_o = 2 * blocks * nt * 8 * head_dim * sizeof(float);
  z.part_ml = 2 * blocks * nt * 8 * sizeof(float2);
  z.desc = (blocks * sizeof(int4) + 255) & ~(size_t)255;
  return z;
}

const char* ca_check_heads(int n_q_heads, int n_kv_heads, int head_dim, int n_q_tokens) {
  if (head_dim != 64 && head_dim != 128) return "head_dim must be 64 or 128";
  if (n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads) return "n_q_heads must be a multiple of n_kv_heads";
  if (n_q_tokens < 1 || n_q_tokens > 64) return "n_q_tokens must be in [1, 64]";
  if (n_q_heads / n_kv_heads > 1024) return "more than 1024 query heads per KV head";
  return nullptr;
}

}  // namespace

extern "C" size_t dd_cache_decode_attn_workspace(int n_q_heads, int n_kv_heads, int head_dim, int n_q_tokens) {
  if (ca_check_heads(n_q_heads, n_kv_heads, head_dim, n_q_tokens)) return 0;
  return ca_size(head_dim, n_q_tokens * (n_q_heads / n_kv_heads), ca_sm_count()).total();
}

extern "C" int dd_cache_decode_attn(const dd_cache* cache, int n_q_tokens, const dd_rows* q, const int* ctx_len,
                                    const dd_rows* out, float* out_lse, int window, float scale, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  const char* who = "dd_cache_decode_attn";
  DD_TRY(dd_check_cache(cache, who));
  DD_TRY(dd_check_rows(q, who, "q", cache->head_dim, false));
  DD_TRY(dd_check_rows(out, who, "out", cache->head_dim, true));
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
  a.part_o = (float*)workspace;
  a.part_ml = (float2*)((char*)workspace + z.part_o);
  a.desc = (int4*)((char*)workspace + z.part_o + z.part_ml);
  a.n_q_heads = q->n_heads;
  a.Tq = n_q_tokens;
  a.row_tiles = (a.n_rows + nt * 8 - 1) / (nt * 8);
  a.window = window;
  a.scale_log2 = (float)((scale > 0.f ? (double)scale : 1.0 / sqrt((double)cache->head_dim)) * 1.4426950408889634);
  if ((long long)a.row_tiles * cache->n_kv_heads > 0x7fffffffLL / 64)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: too many heads", who);
  ca_plan p;
  switch (cache->format == DD_CACHE_E4M3 ? (q->dtype == DD_BF16 ? 2 : 3) : (cache->format == DD_CACHE_FP16 ? 1 : 0)) {
    case 0: p = ca_pick<0>(cache->head_dim, nt); break;
    case 1: p = ca_pick<1>(cache->head_dim, nt); break;
    case 2: p = ca_pick<2>(cache->head_dim, nt); break;
    default: p = ca_pick<3>(cache->head_dim, nt); break;
  }
  const int blocks = sms * p.blocks_per_sm;
  DD_CUDA_TRY(nullptr, cudaFuncSetAttribute(p.main_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, p.smem));
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at;
  dd_pdl_attr(&at);
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  cfg.stream = (cudaStream_t)stream;
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(CA_THREADS);
  cfg.dynamicSmemBytes = p.smem;
  void* args[] = {&a};
  DD_CUDA_TRY(nullptr, cudaLaunchKernelExC(&cfg, p.main_kernel, args));
  int max_parts = blocks;
  cfg.gridDim = dim3((unsigned)blocks, (unsigned)(nt * cache->head_dim / 32));
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = (size_t)blocks * 8 * sizeof(float);
  void* jargs[] = {&a, &max_parts};
  DD_CUDA_TRY(nullptr, cudaLaunchKernelExC(&cfg, p.join_kernel, jargs));
  return DD_OK;
}
