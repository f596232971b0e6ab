// Attention of the newest tokens of every request over all of its cached tokens (paged, 16-bit or e4m3 pages).
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
//
// Rounding. A weight enters the second product as two 16-bit parts, its value cut off and the rounded rest (an MMA takes both
// operands in one type): off by 2^-16 relative at most for bf16 pages, by 2^-22 for half pages and half queries, so that the
// output's own rounding is the one that shows. One part (2^-8, 2^-11) left an error of 0.0023 relative on 4096 bf16 tokens where
// the output's rounding alone is 0.00165 (half: 0.00028 for 0.00021). The second part costs 168.1 -> 169.4 us on 8 x 32K tokens
// of bf16, 9.8 -> 10.1 us on 4096, and the same for half. e4m3 pages with bf16 queries go without: half weights (2^-11) are an
// eighth of the output's half step (0.00162 against 0.00161), and the part would cost 369 -> 375 us on 1M tokens. Halves end at
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
// to 32768 tokens e4m3 78-79 us, one request of 4096 tokens 10.0 us (13.2 where the table is 8192 pages wide).
#include "dd_cache.cuh"

namespace {

constexpr int CA_WARPS = 8;
constexpr int CA_THREADS = CA_WARPS * 32;
constexpr int CA_UNIT_COST = 3;              // empty places behind a unit in the flat list
constexpr int CA_WHOLE = 8;                  // a unit of at most so many tiles is not cut: it belongs to the run it begins in
constexpr int CA_MAX_CLUSTER = 8;
constexpr float CA_LAZY = 8.f;               // how far (log2) a weight may exceed the reference
constexpr float CA_NONE = -3.0e38f;          // reference before any token: every finite score exceeds it

// formats: 0 bf16 pages and queries, 1 half pages and queries, 2 / 3 e4m3 pages with bf16 / half queries
template <int FMT> struct ca_types { using Q = __nv_bfloat16; };
template <> struct ca_types<1> { using Q = __half; };
template <> struct ca_types<3> { using Q = __half; };

template <int FMT, int D, int NT>
struct ca_geom {
  static constexpr bool FP8 = FMT >= 2;
  static constexpr int ES = FP8 ? 1 : 2;
  static constexpr int ROW = D * ES;                                  // bytes of a row: 64, 128 or 256
  static constexpr int HALF_BYTES = 16 * ROW;                         // K (or V) of a tile
  // What one copy group of a warp brings: K or V of a tile in turn, or a whole tile where that is small. Halves of 2 KiB keep
  // more in flight (e4m3 at head_dim 128, 8 x 32K tokens: 102 us against 108 with whole tiles), halves of 1 KiB cost more than they
  // bring (head_dim 64: 74 against 63 us), and with the deep ring of two column tiles whole tiles win (126 against 136 us).
  static constexpr bool WHOLE = 2 * HALF_BYTES <= (NT == 1 ? 2048 : 4096);
  static constexpr int EXP_AT = (WHOLE ? 2 : 1) * HALF_BYTES;         // e4m3: exponents of the tile, 16 of K and 16 of V, behind K or all
  static constexpr int SLOT_BYTES = (WHOLE ? 2 : 1) * HALF_BYTES + (FP8 ? 32 : 0);
  static constexpr int COPIES = HALF_BYTES / 512;
  static constexpr int BLOCKS_PER_SM = NT == 1 ? 2 : 1;               // two column tiles need the registers of a whole SM
  static constexpr int RING_BUDGET = (BLOCKS_PER_SM == 2 ? 106 : 212) * 1024;
  static constexpr int STAGES_ = RING_BUDGET / (CA_WARPS * SLOT_BYTES);
  static constexpr int STAGES = STAGES_ > 8 ? 8 : STAGES_;
  // log2 of the factor on P: halves are lifted out of their subnormals; bf16 weights end at 1, so that large values do not
  // leave the range of the fp32 sums.
  static constexpr float HEADROOM = FMT == 0 ? -CA_LAZY : 6.f;
  // Weights as two 16-bit parts (see "Rounding").
  static constexpr bool PAIR = FMT != 2;
  // A second copy of the tile's code without masks and questions: 131 -> 111 us (128 query heads, 8 x 32K tokens e4m3), 63 -> 58
  // (head_dim 64), 106 -> 104 (e4m3, head_dim 128). bf16 and half pages with one column tile at head_dim 128 wait for memory with
  // either and go without.
  static constexpr bool PLAIN_LOOP = FP8 || NT == 2 || D == 64;
  static constexpr int WARP_BYTES = STAGES * SLOT_BYTES;
  static constexpr int QUADS = NT * (D / 16) * 32;                    // groups of four accumulators: [column tile][product][lane]
  // behind the rings, for clusters: what a block receives of its slice of the quads, and every block's references and sums
  static constexpr int RECV_AT = CA_WARPS * WARP_BYTES;
  static constexpr int RECV_ML_AT = RECV_AT + QUADS * 16;
  static constexpr int SMEM_CLUSTER = RECV_ML_AT + CA_MAX_CLUSTER * NT * 8 * 8;
  static constexpr int SMEM = CA_WARPS * WARP_BYTES;
  static constexpr int NACC = D / 4;                                  // accumulator registers per column tile
  static_assert(WARP_BYTES >= NT * NACC * 128, "a warp's ring holds its accumulators at the end");
};

// Byte offset of 16-byte chunk c of row r in a half tile: a column of 8 rows covers all 32 banks.
template <int ROW> __device__ __forceinline__ uint32_t ca_place(int r, int c) {
  if (ROW >= 128) return r * ROW + ((c ^ (r & 7)) << 4);
  return r * ROW + ((c ^ ((r >> 1) & 3)) << 4);                       // 64-byte rows: two of them make a line
}

struct ca_args {
  dd_cache_view c;
  const char* q;
  char* out;
  long long q_token_stride, q_head_stride, out_token_stride, out_head_stride;   // bytes
  const int* ctx_len;
  float* lse;
  float4* part_o;      // [2 * warps][NT][D / 16][32]
  float2* part_ml;     // [2 * warps][NT * 8]
  int4* desc;          // [warps]: (request, sub, last run + 1) of the cut unit that begins in a warp's run, or 0
  int n_q_heads, G, Tq, n_rows, row_tiles, window;
  int cluster;         // blocks of a cluster that share one unit, 0 = the flat list
  int joins;           // the joining kernel follows
  uint32_t by_G;       // ceil(2^31 / G): row / G by a multiplication
  float scale_log2;
};

__device__ __forceinline__ void ca_cp16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ca_cp4(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ca_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void ca_cp4_all(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
template <int N> __device__ __forceinline__ void ca_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ca_ldsm(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ca_ldsm_trans(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ int ca_lds_byte(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return (int)v;
}
// D(16x8, fp32) += A(16x16, row) * B(16x8, col). Not volatile: the compiler may place it where its operands are ready.
template <int FMT>
__device__ __forceinline__ void ca_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (FMT == 0)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The first product of a chain: nothing to add to.
template <int FMT>
__device__ __forceinline__ void ca_mma_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (FMT == 0)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
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
// First parts of two weights, a little below them, so that the rests p - first are positive too and an infinite value times
// either part is that infinity (a rest of zero would make it NaN). Zero gives zero. The differences are exact in fp32.
template <typename T> __device__ __forceinline__ uint32_t ca_first_part(float p0, float p1);
template <> __device__ __forceinline__ uint32_t ca_first_part<__nv_bfloat16>(float p0, float p1) {
  constexpr float below = 1.f - 0x1p-16f;                              // then cut off
  return __byte_perm(__float_as_uint(p0 * below), __float_as_uint(p1 * below), 0x7632u);
}
template <> __device__ __forceinline__ uint32_t ca_first_part<__half>(float p0, float p1) {
  constexpr float below = 1.f - 0x1p-22f, least = 0x1p-24f - 0x1p-32f; // just under the smallest half; then cut off
  uint32_t r;
  asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(fmaf(p1, below, -least)), "f"(fmaf(p0, below, -least)));
  return r;
}
__device__ __forceinline__ void ca_cp16_all(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// What adding the rows of i copies of 512 bytes changes in ca_place's xor.
template <int ROW> __device__ __forceinline__ constexpr uint32_t ca_twist(int i) {
  return ROW >= 128 ? ((i * (512 / ROW)) & 7) << 4 : 0;              // 64-byte rows: 8 rows a copy, nothing changes
}
__device__ __forceinline__ long long ca_div(long long x, int y) {    // x >= 0, y > 0
  return (x >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)y) : x / y;
}

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

// Query token of row r < 2^16 of a unit (r / G, exact for G <= 1024), and a unit's row tile.
__device__ __forceinline__ int ca_token(const ca_args& a, int r) { return (int)__umulhi((uint32_t)r << 1, a.by_G); }
__device__ __forceinline__ int ca_row_tile(const ca_args& a, int sub) { return a.row_tiles == 1 ? 0 : sub / a.c.n_kv_heads; }

// A place in the flat list: tile t of unit (b, sub), `left` places before the end of the run.
struct ca_cursor {
  int b, sub, t, left;   // sub = row tile * heads + head
  ca_span s;
};
// At the first tile of a unit: the run takes all of it where it is short.
__device__ __forceinline__ void ca_keep_whole(ca_cursor& k) {
  if (k.s.tiles <= CA_WHOLE && k.left < k.s.tiles) k.left = k.s.tiles;
}
// To the first tile of the next unit.
__device__ __forceinline__ void ca_next_unit(const ca_args& a, ca_cursor& k, int subs) {
  k.t = 0;
  if (++k.sub == subs) {
    k.sub = 0;
    do {
      if (k.b + 1 >= a.c.batch) { k.left = 0; return; }
      k.s = ca_span_of(a, ++k.b, false);
    } while (k.s.tiles == 0);
  }
  ca_keep_whole(k);
}
__device__ __forceinline__ void ca_step(const ca_args& a, ca_cursor& k, int subs) {
  --k.left;
  if (++k.t >= k.s.tiles) {
    k.left -= CA_UNIT_COST;
    if (k.left > 0) ca_next_unit(a, k, subs);
  }
}

// Channel of accumulator m at row g of the product (row g + 8: + ca_pair).
__device__ __forceinline__ int ca_channel(bool fp8, int g, int m) { return 16 * m + (fp8 ? 2 * g : g); }
__device__ __forceinline__ constexpr int ca_pair(bool fp8) { return fp8 ? 1 : 8; }

// Two neighbouring results of a query row (accumulator m, rows g and g + 8 of the product) to the row's output.
template <bool FP8> __device__ __forceinline__ void ca_store(char* row, int g, int m, uint32_t w) {
  if (FP8) {
    *reinterpret_cast<uint32_t*>(row + 2 * ca_channel(FP8, g, m)) = w;
  } else {
    *reinterpret_cast<unsigned short*>(row + 2 * ca_channel(FP8, g, m)) = (unsigned short)w;
    *reinterpret_cast<unsigned short*>(row + 2 * (ca_channel(FP8, g, m) + ca_pair(FP8))) = (unsigned short)(w >> 16);
  }
}
// x += v * (scale of the column): elements 0 and 2 belong to the lane's first column, 1 and 3 to its second
__device__ __forceinline__ void ca_add(float4& x, const float4& v, float s0, float s1) {
  x.x = fmaf(v.x, s0, x.x);
  x.y = fmaf(v.y, s1, x.y);
  x.z = fmaf(v.z, s0, x.z);
  x.w = fmaf(v.w, s1, x.w);
}

__device__ __forceinline__ float ca_lse(float from, float den) { return (from + log2f(den)) * 0.6931471805599453f; }

template <int FMT, int D, int NT>
__global__ void __launch_bounds__(CA_THREADS, (ca_geom<FMT, D, NT>::BLOCKS_PER_SM)) dd_cache_attn_kernel(const ca_args a) {
  using geo = ca_geom<FMT, D, NT>;
  constexpr bool PLAIN_LOOP = geo::PLAIN_LOOP;
  using TQ = typename ca_types<FMT>::Q;
  using TP = typename ca_types<FMT == 0 ? 0 : 1>::Q;
  constexpr bool FP8 = geo::FP8;
  constexpr int NS = geo::STAGES;
  extern __shared__ __align__(128) unsigned char ca_smem[];
  __shared__ float2 sh_ml[CA_WARPS][NT * 8];
  __shared__ float sh_scale[CA_WARPS][NT * 8];
  __shared__ float2 sh_blk[NT * 8];                  // clusters: the block's references and sums
  __shared__ int4 sh_rest[CA_WARPS][2];              // the using cursor, while the registers are needed for the tiles
  __shared__ int2 sh_piece[CA_WARPS];                // (request, sub) of the unit a run ends inside, or -1

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  const int subs = a.row_tiles * a.c.n_kv_heads;
  const int B = a.c.batch;
  const int me = blockIdx.x * CA_WARPS + warp;

  dd_grid_dependency_wait();
  // the joining kernel's blocks may take the places that this grid's blocks leave (each waits for all of them). No signal for
  // any other kernel: append and attention in turn, 8 requests of 100 tokens, 14.0 us a layer with one, 12.9 without
  if (a.joins) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  ca_cursor is;
  is.b = is.sub = is.t = is.left = 0;
  long long share = 1;
  if (a.cluster) {
    // ---- one unit per cluster, cut evenly among its warps
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // waited for before the first write into a peer
    const int unit = blockIdx.x / a.cluster, w = blockIdx.x % a.cluster * CA_WARPS + warp;
    is.b = unit / subs;
    is.sub = unit - is.b * subs;
    is.s = ca_span_of(a, is.b, is.sub == 0 && w == 0);
    const int each = (is.s.tiles + a.cluster * CA_WARPS - 1) / (a.cluster * CA_WARPS);
    is.t = each * w;
    is.left = max(0, min(each, is.s.tiles - is.t));
  } else {
    // ---- this warp's run of the flat list: every warp adds up the list by itself, 32 requests at a time
    is.s = ca_span_of(a, min(lane, B - 1), blockIdx.x == 0 && warp == 0 && lane < B);
    auto places = [&](const ca_span& sp) -> long long { return sp.tiles > 0 ? (long long)(sp.tiles + CA_UNIT_COST) * subs : 0; };
    const long long cost0 = lane < B ? places(is.s) : 0;               // of the first 32 requests
    long long total = cost0;
    for (int b = lane + 32; b < B; b += 32) total += places(ca_span_of(a, b, blockIdx.x == 0 && warp == 0));
#pragma unroll
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    share = max(1LL, ca_div(total + (long long)gridDim.x * CA_WARPS - 1, (int)gridDim.x * CA_WARPS));
    const long long f0 = share * me;
    if (f0 < total) {
      long long at = 0;                                                 // first place of the 32 requests looked at
      for (int b0 = 0;; b0 += 32) {
        ca_span sp = is.s;
        long long cost = cost0;
        if (b0 > 0) {
          sp = ca_span_of(a, min(b0 + lane, B - 1), false);
          cost = b0 + lane < B ? places(sp) : 0;
        }
        long long incl = cost;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const long long v = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += v;
        }
        const unsigned in = __ballot_sync(0xffffffffu, f0 >= at + incl - cost && f0 < at + incl);
        if (in) {
          const int l = __ffs(in) - 1;
          is.b = b0 + l;
          is.s.end = __shfl_sync(0xffffffffu, sp.end, l);
          is.s.first = __shfl_sync(0xffffffffu, sp.first, l);
          is.s.tile0 = __shfl_sync(0xffffffffu, sp.tile0, l);
          is.s.tiles = __shfl_sync(0xffffffffu, sp.tiles, l);
          const long long off = f0 - (at + __shfl_sync(0xffffffffu, incl - cost, l));
          is.sub = (int)ca_div(off, is.s.tiles + CA_UNIT_COST);
          is.t = (int)(off - (long long)is.sub * (is.s.tiles + CA_UNIT_COST));
          is.left = (int)min(share, 0x7fffffffLL);
          break;
        }
        at += __shfl_sync(0xffffffffu, incl, 31);
        if (b0 + 32 >= B) break;                                        // lengths changed under the call
      }
      if (is.left > 0 && is.t == 0) {
        ca_keep_whole(is);
      } else if (is.left > 0 && (is.t >= is.s.tiles || is.s.tiles <= CA_WHOLE)) {
        // the run begins in the empty places behind a unit, or inside a short one, which is the run before's
        is.left -= is.s.tiles + CA_UNIT_COST - is.t;
        if (is.left > 0) ca_next_unit(a, is, subs);
      }
    }
  }

  // ---- the issuing side
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ca_smem) + warp * geo::WARP_BYTES;
  ca_cursor u = is;                                  // the using side starts at the same place
  const int page_mask = (1 << a.c.page_shift) - 1;
  // Table entries of the next 32 tiles of the unit, one per lane.
  int blocks = 0, blocks_from = 0, blocks_of = -1;   // entries at hand, the first one's tile, their request
  const char* head_at = nullptr;                     // page 0 of the unit's head
  auto look_up = [&]() {
    blocks_from = is.t;
    blocks_of = is.b;
    const int i = min(is.t + lane, is.s.tiles - 1);
    blocks = __ldg(a.c.table + is.b * a.c.table_stride + (((is.s.tile0 + i) << 4) >> a.c.page_shift));
  };
  auto all_good = [&]() { return __all_sync(0xffffffffu, (unsigned)blocks < (unsigned)a.c.n_blocks); };
  auto enter_unit = [&]() {
    const int rt = ca_row_tile(a, is.sub), head = is.sub - rt * a.c.n_kv_heads;
    head_at = a.c.data + head * a.c.head_stride;
    // the next head of the same request has the same table: short units would wait for it anew at every head
    if (blocks_of != is.b || blocks_from != 0 || is.t != 0) look_up();
    // The unit's query rows are called into L1 a few tiles ahead of their use, every 32-byte sector of them.
    constexpr int SECTORS = D / 16;
#pragma unroll
    for (int i = 0; i < NT * 8 * SECTORS; i += 32) {
      const int row = rt * NT * 8 + (i + lane) / SECTORS;
      if (row < a.n_rows) {
        const int tok = ca_token(a, row);
        const char* at = a.q + ((long long)is.b * a.Tq + tok) * a.q_token_stride + (head * a.G + row - tok * a.G) * a.q_head_stride;
        asm volatile("prefetch.global.L1 [%0];" ::"l"(at + (i + lane) % SECTORS * 32));
      }
    }
  };
  if (is.left > 0) enter_unit();
  const char* src = nullptr;                         // K of the tile being issued; V lies page_tokens rows behind
  int n_first = 0, n_valid = 0;                      // tokens [n_first, n_valid) of it exist (and are visible to some row)
  uint32_t put = ring;                               // slot it goes to
  const uint32_t place0 = ca_place<geo::ROW>(lane / (geo::ROW / 16), lane % (geo::ROW / 16));

  // Copy i of a half takes bytes [512 i, 512 i + 512): 8, 4 or 2 rows; its row numbers change the swizzle by a constant.
  auto copy_full = [&](uint32_t to, const char* from) {
#pragma unroll
    for (int i = 0; i < geo::COPIES; ++i)
      ca_cp16_all(to + (place0 ^ ca_twist<geo::ROW>(i)) + i * 512, from + i * 512 + lane * 16);
  };
  auto copy_half = [&](uint32_t to, const char* from) {
    if (n_first <= 0 && n_valid >= 16) {
      copy_full(to, from);
    } else {
#pragma unroll
      for (int i = 0; i < geo::COPIES; ++i) {
        const int r = i * (512 / geo::ROW) + lane / (geo::ROW / 16);
        ca_cp16(to + (place0 ^ ca_twist<geo::ROW>(i)) + i * 512, from + i * 512 + lane * 16, (r >= n_first && r < n_valid) ? 16u : 0u);
      }
    }
  };
  auto issue = [&](bool v_half) {                    // K (or everything) of the tile at hand, or its V, which ends it
    if (is.left > 0) {
      if (geo::WHOLE || !v_half) {
        const int tok0 = (is.s.tile0 + is.t) << 4;
        int blk = __shfl_sync(0xffffffffu, blocks, is.t - blocks_from);
        n_first = is.s.first - tok0;
        n_valid = is.s.end - tok0;
        if ((unsigned)blk >= (unsigned)a.c.n_blocks) {
          if (lane == 0) dd_status(a.c.status, blk);
          blk = 0;
          n_valid = 0;                               // reads as zeros
        }
        const int in_page = tok0 & page_mask;
        const char* page = head_at + blk * a.c.block_stride;
        src = page + in_page * geo::ROW;
        copy_half(put, src);
        if (FP8 && lane < 8) {
          // exponents: K's behind all the codes of the page, V's behind those
          const char* ex = page + (2 * D + (lane >> 2)) * (page_mask + 1) + in_page + (lane & 3) * 4;
          ca_cp4(put + geo::EXP_AT + lane * 4, ex, n_valid > 0 ? 4u : 0u);
        }
      }
      if (geo::WHOLE || v_half) {
        copy_half(put + (geo::WHOLE ? geo::HALF_BYTES : 0), src + (page_mask + 1) * geo::ROW);
        ca_step(a, is, subs);
        if (is.left > 0) {
          if (is.t == 0) enter_unit();
          else if (is.t - blocks_from == 32) look_up();
        }
      }
    }
    ca_commit();
    put = put + geo::SLOT_BYTES == ring + geo::WARP_BYTES ? ring : put + geo::SLOT_BYTES;
  };
#pragma unroll 1
  for (int i = 0; i < NS; ++i) issue(i & 1);
  // The same inside a unit, where nothing has to be asked: a complete tile of a good block, not the last of the run, the unit
  // or the entries at hand. First half of a pair: V of the tile at hand if the ring's depth is odd, else K (or everything) of it.
  constexpr bool V_FIRST = !geo::WHOLE && (NS & 1);
  auto plain_k = [&]() {
    const int in_page = ((is.s.tile0 + is.t) << 4) & page_mask;
    const char* page = head_at + __shfl_sync(0xffffffffu, blocks, is.t - blocks_from) * a.c.block_stride;
    src = page + in_page * geo::ROW;
    copy_full(put, src);
    if (FP8 && lane < 8) ca_cp4_all(put + geo::EXP_AT + lane * 4, page + (2 * D + (lane >> 2)) * (page_mask + 1) + in_page + (lane & 3) * 4);
    if (geo::WHOLE) copy_full(put + geo::HALF_BYTES, src + (page_mask + 1) * geo::ROW);
  };
  auto plain_v = [&]() { copy_full(put, src + (page_mask + 1) * geo::ROW); };
  auto next_put = [&]() {
    ca_commit();
    put = put + geo::SLOT_BYTES == ring + geo::WARP_BYTES ? ring : put + geo::SLOT_BYTES;
  };
  auto issue_plain = [&](bool first) {
    if (first != V_FIRST) {
      plain_k();
    } else {
      plain_v();
    }
    if (geo::WHOLE || first == V_FIRST) {            // the tile is complete: on to the next
      ++is.t;
      --is.left;
    }
    next_put();
  };
  uint32_t take = ring;                              // slot of the next copy group to use
  auto use_up = [&](bool plain, bool first) {        // everything of the slot is in registers: refill it
    __syncwarp();
    take = take + geo::SLOT_BYTES == ring + geo::WARP_BYTES ? ring : take + geo::SLOT_BYTES;
    if (plain) issue_plain(first);
    else issue(first == V_FIRST);
  };
  // ldmatrix addresses: K matrices (rows 0-7 | 8-15) x (chunk 2i | 2i+1), V matrices the same or with the two swapped
  const int r8 = lane & 7, m1 = (lane >> 3) & 1, m2 = lane >> 4;
  const uint32_t k_row = (r8 + 8 * m1) * geo::ROW, k_x = (ca_place<geo::ROW>(r8 + 8 * m1, 0) - k_row) ^ (m2 << 4);
  const int v_r = FP8 ? r8 + 8 * m1 : r8 + 8 * m2, v_c = FP8 ? m2 : m1;
  const uint32_t v_row = v_r * geo::ROW, v_x = (ca_place<geo::ROW>(v_r, 0) - v_row) ^ (v_c << 4);

  // ---- the using side, unit by unit
  int4 desc = make_int4(0, 0, 0, 0);
  int2 inside = make_int2(-1, 0);
  float acc[NT][D / 16][4];
  float from[NT][2], sum[NT][2];                     // reference minus headroom; denominator, this lane's tokens
  while (u.left > 0) {
    int b = u.b, sub = u.sub, t0 = u.t;
    ca_span s = u.s;
    int n_here = min(s.tiles - t0, u.left);                           // tiles of the unit in this run
    if (n_here <= 0) break;                                           // lengths changed under the call: stop
    int rt = ca_row_tile(a, sub), head = sub - rt * a.c.n_kv_heads;
    int r0 = rt * NT * 8;                                       // first row of the tile

    // query fragments: column n = g of column tile nt is row r0 + 8 nt + g
    uint32_t qf[NT][D / 8];
    float zs[NT][2];
    int pos[NT][2];                                                   // position of the lane's two columns, -1 = no such row
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = r0 + nt * 8 + g;
      if (row < a.n_rows) {
        const int tok = ca_token(a, row);
        const char* qr = a.q + ((long long)b * a.Tq + tok) * a.q_token_stride + (head * a.G + row - tok * a.G) * a.q_head_stride;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          if (FP8) {                                                  // k-slots 2t, 2t+1 | 2t+8, 2t+9: channels 4t .. 4t+3 of 16
            const uint2 w = *reinterpret_cast<const uint2*>(qr + 2 * (16 * ks + 4 * t));
            qf[nt][2 * ks] = w.x;
            qf[nt][2 * ks + 1] = w.y;
          } else {
            qf[nt][2 * ks] = *reinterpret_cast<const uint32_t*>(qr + 2 * (16 * ks + 2 * t));
            qf[nt][2 * ks + 1] = *reinterpret_cast<const uint32_t*>(qr + 2 * (16 * ks + 8 + 2 * t));
          }
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < D / 8; ++ks) qf[nt][ks] = 0u;
      }
      float back = 1.f;                                               // what the row was divided by
      if (FP8) {
        float amax = 0.f;
#pragma unroll
        for (int ks = 0; ks < D / 8; ++ks) {
          const float2 w = dd_unpack2<TQ>(qf[nt][ks]);
          amax = fmaxf(amax, fmaxf(fabsf(w.x), fabsf(w.y)));
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
        for (int ks = 0; ks < D / 8; ++ks) {
          const float2 w = dd_unpack2<TQ>(qf[nt][ks]);
          qf[nt][ks] = dd_pack2<__half>(w.x * by, w.y * by);
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        zs[nt][c] = a.scale_log2 * (FP8 ? __shfl_sync(0xffffffffu, back, (2 * t + c) * 4) : 1.f);
        const int r = r0 + nt * 8 + 2 * t + c;
        pos[nt][c] = r < a.n_rows ? s.end - a.Tq + ca_token(a, r) : -1;
      }
    }
    const int pos_lo = s.end - a.Tq + ca_token(a, r0);                       // positions of the first and last row of the tile
    const int pos_hi = s.end - a.Tq + ca_token(a, min(a.n_rows, r0 + NT * 8) - 1);

#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int m = 0; m < D / 16; ++m) acc[nt][m][0] = acc[nt][m][1] = acc[nt][m][2] = acc[nt][m][3] = 0.f;
      from[nt][0] = from[nt][1] = CA_NONE;
      sum[nt][0] = sum[nt][1] = 0.f;
    }

    const int first_tile = s.tile0 + t0;
    if (lane == 0) {
      sh_rest[warp][0] = make_int4(u.b, u.sub, u.t, u.left);
      sh_rest[warp][1] = make_int4(s.end, s.first, s.tile0, s.tiles);
    }
    __syncwarp();
    auto tile = [&](auto plain_, int i) {
      constexpr bool plain = decltype(plain_)::value;                 // no mask, and the refills need no questions
      const int tok0 = (first_tile + i) << 4;
      // ---- scores
      float z[NT][4];
      float vex0 = 0.f, vex1 = 0.f;                                   // log2 of the value scales of tokens g, g + 8
      ca_wait<NS - 1>();
      __syncwarp();
      {
        float z2[NT][4];                                              // two chains: the products of one depend on each other
        const uint32_t at = take + k_row;
        float by0 = 1.f, by1 = 1.f;                                   // key scales of tokens g, g + 8
        if (FP8) {
          // byte 0 stands for 2^-127, whose bits lie below those of all the others
          by0 = __uint_as_float(max((uint32_t)ca_lds_byte(take + geo::EXP_AT + g) << 23, 0x00400000u));
          by1 = __uint_as_float(max((uint32_t)ca_lds_byte(take + geo::EXP_AT + g + 8) << 23, 0x00400000u));
          vex0 = (float)(ca_lds_byte(take + geo::EXP_AT + 16 + g) - 127);
          vex1 = (float)(ca_lds_byte(take + geo::EXP_AT + 16 + g + 8) - 127);
          uint32_t r[D / 32][4];                                      // four codes each: rows g, g + 8 of chunk 2c, of chunk 2c + 1
#pragma unroll
          for (int c = 0; c < D / 32; ++c) ca_ldsm(r[c], at + (k_x ^ (c << 5)));
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              uint32_t a0, a1, a2, a3;
              dd_e4m3x4_to_half(r[c][2 * w], a0, a2);
              dd_e4m3x4_to_half(r[c][2 * w + 1], a1, a3);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                if (c == 0) ca_mma_first<FMT>(w ? z2[nt] : z[nt], a0, a1, a2, a3, qf[nt][2 * w], qf[nt][2 * w + 1]);
                else ca_mma<FMT>(w ? z2[nt] : z[nt], a0, a1, a2, a3, qf[nt][4 * c + 2 * w], qf[nt][4 * c + 2 * w + 1]);
              }
            }
          }
        } else {
#pragma unroll
          for (int c4 = 0; c4 < D / 16; c4 += 4) {
            uint32_t r[4][4];
#pragma unroll
            for (int c = 0; c < 4; ++c) ca_ldsm(r[c], at + (k_x ^ ((c4 + c) << 5)));
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                if (c4 + c < 2) ca_mma_first<FMT>((c & 1) ? z2[nt] : z[nt], r[c][0], r[c][1], r[c][2], r[c][3], qf[nt][2 * c], qf[nt][2 * c + 1]);
                else ca_mma<FMT>((c & 1) ? z2[nt] : z[nt], r[c][0], r[c][1], r[c][2], r[c][3], qf[nt][2 * (c4 + c)], qf[nt][2 * (c4 + c) + 1]);
              }
          }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) z[nt][e] = (z[nt][e] + z2[nt][e]) * (FP8 ? zs[nt][e & 1] * (e < 2 ? by0 : by1) : zs[nt][e & 1]);
      }
      if (!geo::WHOLE) use_up(plain, true);
      // whole tiles: V is there already, its first registers come in behind the soft-max
      constexpr int V_LOADS = D / (FP8 ? 32 : 16), V_BATCH = V_LOADS < 4 ? V_LOADS : 4;
      uint32_t raw[V_BATCH][4];
      auto load_values = [&](int c0) {
        const uint32_t at = take + v_row + (geo::WHOLE ? geo::HALF_BYTES : 0);
#pragma unroll
        for (int c = 0; c < V_BATCH; ++c) ca_ldsm_trans(raw[c], at + (v_x ^ ((c0 + c) << 5)));
      };
      if (geo::WHOLE) load_values(0);

      // ---- masks: z[.][0..1] is token tok0 + g, z[.][2..3] token tok0 + g + 8
      const bool partial = !plain && (tok0 + 15 > pos_lo || (a.window > 0 && tok0 <= pos_hi - a.window));
      if (partial) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int tok = tok0 + g + (e < 2 ? 0 : 8), p = pos[nt][e & 1];
            if (tok > p || (a.window > 0 && tok <= p - a.window)) z[nt][e] = -INFINITY;
          }
      }

      // ---- weights against the reference: 2^x with x = z - ref + headroom for the denominator, + log2 of the value's scale
      // for the product. Weights of values with a scale below 2^-96 do not let the denominator grow out of range: their
      // reference is taken as if the scale were 2^-96.
      uint32_t pb[NT][2], pr[NT][2];                                  // weights, their rests
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float x[4], y[4];
        bool above = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = z[nt][e] - from[nt][e & 1];
          y[e] = FP8 ? x[e] + (e < 2 ? vex0 : vex1) : x[e];
          above |= y[e] > CA_LAZY + geo::HEADROOM;
          if (FP8) above |= x[e] > CA_LAZY + geo::HEADROOM + 96.f;
        }
        if (__any_sync(0xffffffffu, above)) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float top = FP8 ? fmaxf(z[nt][c] + fmaxf(vex0, -96.f), z[nt][2 + c] + fmaxf(vex1, -96.f)) : fmaxf(z[nt][c], z[nt][2 + c]);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
            top = fmaxf(top - geo::HEADROOM, from[nt][c]);
            const float fix = ca_exp2(from[nt][c] - top);
            from[nt][c] = top;
            sum[nt][c] *= fix;
#pragma unroll
            for (int m = 0; m < D / 16; ++m) { acc[nt][m][c] *= fix; acc[nt][m][2 + c] *= fix; }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[e] = z[nt][e] - from[nt][e & 1];
            y[e] = FP8 ? x[e] + (e < 2 ? vex0 : vex1) : x[e];
          }
        }
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[e] = ca_exp2(y[e]);
          sum[nt][e & 1] += FP8 ? ca_exp2(x[e]) : p[e];
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (geo::PAIR) {
            const uint32_t w = ca_first_part<TP>(p[2 * k], p[2 * k + 1]);
            const float2 had = dd_unpack2<TP>(w);
            pb[nt][k] = ca_transpose(w);
            pr[nt][k] = ca_transpose(dd_pack2<TP>(p[2 * k] - had.x, p[2 * k + 1] - had.y));
          } else {
            pb[nt][k] = ca_transpose(dd_pack2<TP>(p[2 * k], p[2 * k + 1]));
          }
        }
      }

      // ---- weighted values
      if (!geo::WHOLE) {
        ca_wait<NS - 1>();
        __syncwarp();
      }
      // Registers of V^T: r[0], r[1] hold tokens 2t | 2t+1 (low | high half), r[2], r[3] tokens 2t+8 | 2t+9, for the channels of
      // rows g and g + 8.
      auto value_frag = [&](uint32_t (&r)[4], const uint32_t (&v)[4], int half) {
        if (FP8) {
          // bytes of a register: two channels of token 2t, the same two of 2t+1; token pairs side by side, then as halves
          dd_e4m3x4_to_half(__byte_perm(v[2 * half], 0u, 0x3120u), r[0], r[1]);
          dd_e4m3x4_to_half(__byte_perm(v[2 * half + 1], 0u, 0x3120u), r[2], r[3]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) r[e] = v[e];
        }
      };
      if (!(partial && a.Tq > 1)) {
#pragma unroll
        for (int c0 = 0; c0 < V_LOADS; c0 += V_BATCH) {
          if (!geo::WHOLE || c0 > 0) load_values(c0);
#pragma unroll
          for (int c = 0; c < V_BATCH; ++c)
#pragma unroll
            for (int half = 0; half < (FP8 ? 2 : 1); ++half) {
              uint32_t r[4];
              value_frag(r, raw[c], half);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                ca_mma<FMT>(acc[nt][FP8 ? 2 * (c0 + c) + half : c0 + c], r[0], r[1], r[2], r[3], pb[nt][0], pb[nt][1]);
                if (geo::PAIR) ca_mma<FMT>(acc[nt][FP8 ? 2 * (c0 + c) + half : c0 + c], r[0], r[1], r[2], r[3], pr[nt][0], pr[nt][1]);
              }
            }
        }
      } else {
        // Some tokens are seen by some rows of the tile and not by others: a weight of zero does not keep an infinity or NaN
        // of V out of the sum, so the products are taken query token by query token with the unseen values made zero.
#pragma unroll 1
        for (int p = pos_lo; p <= pos_hi; ++p) {
          uint32_t keep[2];                                           // tokens 2t | 2t+1 and 2t+8 | 2t+9
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int tok = tok0 + 2 * t + 8 * k, first = a.window > 0 ? p - a.window : -1;
            keep[k] = ((tok <= p && tok > first) ? 0xffffu : 0u) | ((tok + 1 <= p && tok + 1 > first) ? 0xffff0000u : 0u);
          }
#pragma unroll
          for (int c0 = 0; c0 < V_LOADS; c0 += V_BATCH) {
            load_values(c0);
#pragma unroll
            for (int c = 0; c < V_BATCH; ++c) {
#pragma unroll
              for (int e = 0; e < 4; ++e) raw[c][e] &= keep[FP8 ? (e & 1) : (e >> 1)];
#pragma unroll
              for (int half = 0; half < (FP8 ? 2 : 1); ++half) {
                uint32_t r[4];
                value_frag(r, raw[c], half);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                  float one[4] = {0.f, 0.f, 0.f, 0.f};
                  ca_mma<FMT>(one, r[0], r[1], r[2], r[3], pb[nt][0], pb[nt][1]);
                  if (geo::PAIR) ca_mma<FMT>(one, r[0], r[1], r[2], r[3], pr[nt][0], pr[nt][1]);
#pragma unroll
                  for (int e = 0; e < 4; ++e)
                    if (pos[nt][e & 1] == p) acc[nt][FP8 ? 2 * (c0 + c) + half : c0 + c][e] += one[e];
                }
              }
            }
          }
        }
      }
      use_up(plain, geo::WHOLE);
    };
    for (int i = 0; i < n_here;) {
      // how many tiles from here are plain on both sides: seen by every row of the tile, and refilled from complete tiles of
      // this lookup, the last of them left to the careful form
      int n = 0;
      if (PLAIN_LOOP && is.left > 1) {
        n = min(min(is.left, blocks_from + 32 - is.t), ((is.s.end - 16) >> 4) - is.s.tile0 - is.t + 1) - 1;
        n = min(n, min(n_here - i, ((pos_lo - 15) >> 4) - (first_tile + i) + 1));
        if (a.window > 0 && (((first_tile + i) << 4) <= pos_hi - a.window || ((is.s.tile0 + is.t) << 4) < is.s.first)) n = 0;
        if (!all_good()) n = 0;
      }
      if constexpr (PLAIN_LOOP) {
#pragma unroll 1
        for (; n > 0; --n, ++i) tile(std::true_type(), i);
      }
      if (i < n_here) tile(std::false_type(), i++);
    }

    // ---- the end of the unit, or of the run
    {
      __syncwarp();
      const volatile int* rest = reinterpret_cast<const volatile int*>(&sh_rest[warp][0]);
      u.b = b = rest[0];
      u.sub = sub = rest[1];
      u.t = t0 = rest[2];
      u.left = rest[3];
      s.end = rest[4];
      s.first = rest[5];
      s.tile0 = rest[6];
      s.tiles = rest[7];
      u.s = s;
      n_here = min(s.tiles - t0, u.left);
      rt = ca_row_tile(a, sub);
      head = sub - rt * a.c.n_kv_heads;
      r0 = rt * NT * 8;
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        sum[nt][c] += __shfl_xor_sync(0xffffffffu, sum[nt][c], 4);
        sum[nt][c] += __shfl_xor_sync(0xffffffffu, sum[nt][c], 8);
        sum[nt][c] += __shfl_xor_sync(0xffffffffu, sum[nt][c], 16);
      }
    const bool ends = t0 + n_here == s.tiles;
    if (a.cluster) break;                                             // one piece a warp
    if (ends && t0 == 0) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int r = r0 + nt * 8 + 2 * t + c;
          if (r < a.n_rows) {
            const int tok = ca_token(a, r), h = head * a.G + r - tok * a.G;
            const long long tn = (long long)b * a.Tq + tok;
            const bool empty = pos[nt][c] < 0;
            const float inv = empty ? 0.f : __frcp_rn(sum[nt][c]);
            char* o = a.out + tn * a.out_token_stride + h * a.out_head_stride;
#pragma unroll
            for (int m = 0; m < D / 16; ++m) ca_store<FP8>(o, g, m, empty ? 0u : dd_pack2<TQ>(acc[nt][m][c] * inv, acc[nt][m][2 + c] * inv));
            if (a.lse && g == 0) a.lse[tn * a.n_q_heads + h] = empty ? -INFINITY : ca_lse(from[nt][c], sum[nt][c]);
          }
        }
    } else if (ends) {                                                // the last piece of a unit that began earlier: slot 2 me
      float4* po = a.part_o + 2LL * me * NT * (D / 16) * 32;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int m = 0; m < D / 16; ++m) po[(nt * (D / 16) + m) * 32 + lane] = make_float4(acc[nt][m][0], acc[nt][m][1], acc[nt][m][2], acc[nt][m][3]);
        if (g == 0) {
          a.part_ml[2LL * me * NT * 8 + nt * 8 + 2 * t] = make_float2(from[nt][0], sum[nt][0]);
          a.part_ml[2LL * me * NT * 8 + nt * 8 + 2 * t + 1] = make_float2(from[nt][1], sum[nt][1]);
        }
      }
    } else {
      inside = make_int2(b, sub);                                     // the run ends here
      if (t0 == 0) desc = make_int4(b, sub, (int)ca_div(share * me + (share - u.left) + s.tiles - 1, (int)share) + 1, 0);
    }

    // ---- the next unit
    u.left -= n_here + CA_UNIT_COST;
    if (u.left > 0) ca_next_unit(a, u, subs);
  }
  if (lane == 0 && !a.cluster) a.desc[me] = desc;
  ca_wait<0>();
  __syncwarp();

  // ---- pieces left over at the ends of the runs: neighbouring warps inside the same unit become one partial, in slot
  // 2 w + 1 of the first of them
  if (a.cluster && u.left <= 0) {                    // a warp without a tile
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int m = 0; m < D / 16; ++m) acc[nt][m][0] = acc[nt][m][1] = acc[nt][m][2] = acc[nt][m][3] = 0.f;
      from[nt][0] = from[nt][1] = CA_NONE;
      sum[nt][0] = sum[nt][1] = 0.f;
    }
  }
  if (a.cluster) inside = make_int2(0, 0);           // all of one unit
  if (lane == 0) sh_piece[warp] = inside;
  if (inside.x >= 0) {
    float4* own = reinterpret_cast<float4*>(ca_smem + warp * geo::WARP_BYTES);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int m = 0; m < D / 16; ++m) own[(nt * (D / 16) + m) * 32 + lane] = make_float4(acc[nt][m][0], acc[nt][m][1], acc[nt][m][2], acc[nt][m][3]);
      if (g == 0) {
        sh_ml[warp][nt * 8 + 2 * t] = make_float2(from[nt][0], sum[nt][0]);
        sh_ml[warp][nt * 8 + 2 * t + 1] = make_float2(from[nt][1], sum[nt][1]);
      }
    }
  }
  // units without a token: zeros and -inf, shared out over the blocks
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
  __syncthreads();
  auto same = [&](int v, int w) { return sh_piece[v].x == sh_piece[w].x && sh_piece[v].y == sh_piece[w].y; };
  auto chain_end = [&](int w0) {                     // warps w0 .. w1 - 1 hold pieces of one unit
    int w1 = w0 + 1;
    while (w1 < CA_WARPS && same(w1, w0)) ++w1;
    return w1;
  };
  for (int i = threadIdx.x; i < CA_WARPS * NT * 8; i += CA_THREADS) {
    const int w = i / (NT * 8), row = i % (NT * 8);
    if (sh_piece[w].x < 0) continue;
    int w0 = w;
    while (w0 > 0 && same(w0 - 1, w)) --w0;
    const int w1 = chain_end(w0);
    float M = CA_NONE, L = 0.f;
    for (int v = w0; v < w1; ++v) M = fmaxf(M, sh_ml[v][row].x);
    for (int v = w0; v < w1; ++v) L = fmaf(sh_ml[v][row].y, ca_exp2(sh_ml[v][row].x - M), L);
    sh_scale[w][row] = ca_exp2(sh_ml[w][row].x - M);
    if (w == w0 && a.cluster) sh_blk[row] = make_float2(M, L);
    else if (w == w0) a.part_ml[(2LL * (blockIdx.x * CA_WARPS + w0) + 1) * NT * 8 + row] = make_float2(M, L);
  }
  __syncthreads();
  constexpr int QUADS = geo::QUADS;
  if (a.cluster) {
    // ---- the blocks of a cluster: block r owns a slice of the quads; every block sends it its part of them (remote stores, nobody
    // waits for an answer), one barrier makes them visible, and every block adds and writes its slice
    const int C = a.cluster, slice = QUADS / C, rank = blockIdx.x % C;
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    const uint32_t recv = (uint32_t)__cvta_generic_to_shared(ca_smem) + geo::RECV_AT, recv_ml = (uint32_t)__cvta_generic_to_shared(ca_smem) + geo::RECV_ML_AT;
    for (int e = threadIdx.x; e < QUADS; e += CA_THREADS) {
      const int row = e / (D / 16 * 32) * 8 + 2 * (e & 3);
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < CA_WARPS; ++w)
        ca_add(x, reinterpret_cast<const float4*>(ca_smem + w * geo::WARP_BYTES)[e], sh_scale[w][row], sh_scale[w][row + 1]);
      uint32_t to;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(recv + (rank * slice + e % slice) * 16), "r"(e / slice));
      asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to), "f"(x.x), "f"(x.y), "f"(x.z), "f"(x.w) : "memory");
    }
    for (int i = threadIdx.x; i < C * NT * 8; i += CA_THREADS) {
      const float2 ml = sh_blk[i % (NT * 8)];
      uint32_t to;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(recv_ml + (rank * NT * 8 + i % (NT * 8)) * 8), "r"(i / (NT * 8)));
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(ml.x), "f"(ml.y) : "memory");
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    const float4* in = reinterpret_cast<const float4*>(ca_smem + geo::RECV_AT);
    const float2* in_ml = reinterpret_cast<const float2*>(ca_smem + geo::RECV_ML_AT);
    for (int i = threadIdx.x; i < slice; i += CA_THREADS) {
      const int e = rank * slice + i, row = e / (D / 16 * 32) * 8 + 2 * (e & 3);
      float M[2] = {CA_NONE, CA_NONE}, L[2] = {0.f, 0.f};
      for (int k = 0; k < C; ++k) {
        M[0] = fmaxf(M[0], in_ml[k * NT * 8 + row].x);
        M[1] = fmaxf(M[1], in_ml[k * NT * 8 + row + 1].x);
      }
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k = 0; k < C; ++k) {
        const float2 m0 = in_ml[k * NT * 8 + row], m1 = in_ml[k * NT * 8 + row + 1];
        const float s0 = ca_exp2(m0.x - M[0]), s1 = ca_exp2(m1.x - M[1]);
        L[0] = fmaf(m0.y, s0, L[0]);
        L[1] = fmaf(m1.y, s1, L[1]);
        ca_add(x, in[k * slice + i], s0, s1);
      }
      const int unit = blockIdx.x / C, b = unit / subs, sub = unit - b * subs;
      const int rt = ca_row_tile(a, sub), head = sub - rt * a.c.n_kv_heads, m = (e / 32) % (D / 16), ge = (e & 31) >> 2;
      const ca_span s = ca_span_of(a, b, false);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int r = rt * NT * 8 + row + c;
        if (r < a.n_rows && s.tiles > 0) {           // (a request without a token has been written above)
          const int tok = ca_token(a, r), h = head * a.G + r - tok * a.G;
          const long long tn = (long long)b * a.Tq + tok;
          const bool empty = s.end - a.Tq + tok < 0;
          const float lo = c ? x.y : x.x, hi = c ? x.w : x.z;
          ca_store<FP8>(a.out + tn * a.out_token_stride + h * a.out_head_stride, ge, m, empty ? 0u : dd_pack2<TQ>(lo / L[c], hi / L[c]));
          if (a.lse && m == 0 && ge == 0) a.lse[tn * a.n_q_heads + h] = empty ? -INFINITY : ca_lse(M[c], L[c]);
        }
      }
    }
    return;
  }
  for (int w0 = 0, w1; w0 < CA_WARPS; w0 = w1) {
    w1 = w0 + 1;
    if (sh_piece[w0].x < 0) continue;
    w1 = chain_end(w0);
    float4* po = a.part_o + (2LL * (blockIdx.x * CA_WARPS + w0) + 1) * QUADS;
    for (int e = threadIdx.x; e < QUADS; e += CA_THREADS) {
      const int row = e / (D / 16 * 32) * 8 + 2 * (e & 3);
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < CA_WARPS; ++w)
        if (w >= w0 && w < w1) ca_add(x, reinterpret_cast<const float4*>(ca_smem + w * geo::WARP_BYTES)[e], sh_scale[w][row], sh_scale[w][row + 1]);
      po[e] = x;
    }
  }

}

// Adds the partials of the cut units that begin in the attention kernel's runs x, x + gridDim.x, ... The partials of a unit from run w0
// (where it begins) to run w1 (where it ends) are one per block among the runs w0 .. w1 - 1, in the slot of the first of
// them, and the last piece. Grid (blocks of the attention kernel, groups of 64 quads of accumulators); four groups of
// threads take every fourth partial of the same 64 quads. What bounds it is latency: (descriptors) -> (references, sums,
// the first 32 partials, the length) -> result.
constexpr int CJ_GROUPS = 4;
template <int FMT, int D, int NT>
__global__ void __launch_bounds__(64 * CJ_GROUPS) dd_cache_attn_join_kernel(const ca_args a) {
  using TQ = typename ca_types<FMT>::Q;
  constexpr bool FP8 = FMT >= 2;
  constexpr int QUADS = NT * (D / 16) * 32;
  constexpr int AHEAD = 8;                                            // partials of a group fetched before the scales are known
  extern __shared__ float cj_scale[];                                 // [parts][8] of the column tile
  __shared__ float2 sh_ml[8];
  __shared__ float4 sh_x[CJ_GROUPS][64];
  const int q = threadIdx.x & 63, grp = threadIdx.x >> 6;
  const int e = blockIdx.y * 64 + q;                                  // quad: [column tile][product][lane]
  const int nt = blockIdx.y * 64 / (D / 16 * 32), m = (e / 32) % (D / 16), ge = (e & 31) >> 2, col = 2 * (e & 3);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  dd_grid_dependency_wait();
  // every gridDim.x-th descriptor, one per lane, handed round by shuffles (neighbouring ones in different blocks: where units are
  // short, neighbouring runs all have one)
  int4 mine = make_int4(0, 0, 0, 0);
  if (lane < CA_WARPS) mine = a.desc[lane * gridDim.x + blockIdx.x];
  unsigned todo = __ballot_sync(0xffffffffu, mine.z != 0);            // the same in every warp
  while (todo) {
    const int l = __ffs(todo) - 1;
    todo &= todo - 1;
    const int b = __shfl_sync(0xffffffffu, mine.x, l), sub = __shfl_sync(0xffffffffu, mine.y, l);
    const int w0 = l * gridDim.x + blockIdx.x, w1 = __shfl_sync(0xffffffffu, mine.z, l) - 1, first = w0 / CA_WARPS;
    const int n = (w1 - 1) / CA_WARPS - first + 2;                    // partials
    auto slot = [&](int i) -> long long { return i == 0 ? 2LL * w0 + 1 : (i == n - 1 ? 2LL * w1 : 2LL * (first + i) * CA_WARPS + 1); };
    const int end = ca_span_of(a, b, false).end;
    float4 ahead[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (grp + CJ_GROUPS * i < n) ahead[i] = a.part_o[slot(grp + CJ_GROUPS * i) * QUADS + e];
    {
      // warp w: the scales of row w of the column tile
      const int row = nt * 8 + warp;
      const float2 own = lane < n ? a.part_ml[slot(lane) * NT * 8 + row] : make_float2(CA_NONE, 0.f);
      float M = own.x;
      for (int i = lane + 32; i < n; i += 32) M = fmaxf(M, a.part_ml[slot(i) * NT * 8 + row].x);
#pragma unroll
      for (int o = 16; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      const float sc0 = ca_exp2(own.x - M);
      float L = own.y * sc0;
      if (lane < n) cj_scale[lane * 8 + warp] = sc0;
      for (int i = lane + 32; i < n; i += 32) {
        const float2 ml = a.part_ml[slot(i) * NT * 8 + row];
        const float sc = ca_exp2(ml.x - M);
        cj_scale[i * 8 + warp] = sc;
        L = fmaf(ml.y, sc, L);
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
      if (lane == 0) sh_ml[warp] = make_float2(M, L);
    }
    __syncthreads();
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int k = grp + CJ_GROUPS * i;
      if (k < n) ca_add(x, ahead[i], cj_scale[k * 8 + col], cj_scale[k * 8 + col + 1]);
    }
#pragma unroll 8
    for (int k = grp + CJ_GROUPS * AHEAD; k < n; k += CJ_GROUPS)
      ca_add(x, a.part_o[slot(k) * QUADS + e], cj_scale[k * 8 + col], cj_scale[k * 8 + col + 1]);
    sh_x[grp][q] = x;
    __syncthreads();
    if (grp < 2) {                                                    // group c finishes the quads' column c
      const int c = grp;
      float lo = 0.f, hi = 0.f;
#pragma unroll
      for (int k = 0; k < CJ_GROUPS; ++k) {
        const float4 v = sh_x[k][q];
        lo += c ? v.y : v.x;
        hi += c ? v.w : v.z;
      }
      const int rt = sub / a.c.n_kv_heads, head = sub - rt * a.c.n_kv_heads;
      const int r = rt * NT * 8 + nt * 8 + col + c;
      if (r < a.n_rows) {
        const int tok = ca_token(a, r), h = head * a.G + r - tok * a.G;
        const long long tn = (long long)b * a.Tq + tok;
        const bool empty = end - a.Tq + tok < 0;
        const float2 ml = sh_ml[col + c];
        ca_store<FP8>(a.out + tn * a.out_token_stride + h * a.out_head_stride, ge, m, empty ? 0u : dd_pack2<TQ>(lo / ml.y, hi / ml.y));
        if (a.lse && m == 0 && ge == 0) a.lse[tn * a.n_q_heads + h] = empty ? -INFINITY : ca_lse(ml.x, ml.y);
      }
    }
    __syncthreads();                                                  // before the scales are written again
  }
}

struct ca_plan {
  const void* main_kernel;
  const void* join_kernel;
  int smem, smem_cluster, blocks_per_sm;
};
template <int FMT, int D, int NT> ca_plan ca_plan_of() {
  using geo = ca_geom<FMT, D, NT>;
  static_assert(geo::SMEM_CLUSTER + 2048 <= 227 * 1024, "shared memory of a block");
  static_assert(geo::BLOCKS_PER_SM == 1 || geo::SMEM_CLUSTER + 1024 + 2048 <= 114 * 1024, "shared memory of two blocks");
  return {(const void*)dd_cache_attn_kernel<FMT, D, NT>, (const void*)dd_cache_attn_join_kernel<FMT, D, NT>, geo::SMEM, geo::SMEM_CLUSTER, geo::BLOCKS_PER_SM};
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

// Blocks of a cluster per unit, 0 for the flat list. Few and short units (known from the table's width, not from the lengths,
// which are on the device): a cluster per unit joins its pieces through distributed shared memory and needs no second
// kernel and no look at the other requests. At most 8 tiles a warp, and all clusters resident at once; units that fit one warp's
// run uncut are left to the flat list. One request, 8 KV heads, a table of just its pages: 2048 tokens 11.8 -> 8.3 us, 4096
// 13.2 -> 10.0, 8192 14.7 -> 13.6; a table wider than 8192 tokens takes the flat list whatever the length.
int ca_cluster_of(long long units, long long tiles, int blocks) {
  if (tiles <= CA_WHOLE) return 0;
  int c = 2;
  while (c < CA_MAX_CLUSTER && tiles > 2LL * c * CA_WARPS) c *= 2;
  return tiles <= 8LL * c * CA_WARPS && units * c <= blocks * 7 / 8 ? c : 0;
}

// Rows of a unit that go through the MMA together: up to 8 in one column tile, up to 16 in two.
int ca_column_tiles(int rows) { return rows <= 8 ? 1 : 2; }

struct ca_sizes { size_t part_o, part_ml, desc; size_t total() const { return part_o + part_ml + desc; } };
ca_sizes ca_size(int head_dim, int rows, int sms) {
  const int nt = ca_column_tiles(rows);
  const size_t warps = (size_t)sms * (nt == 1 ? 2 : 1) * CA_WARPS;
  ca_sizes z;
  z.part_o = 2 * warps * nt * 8 * head_dim * sizeof(float);
  z.part_ml = 2 * warps * nt * 8 * sizeof(float2);
  z.desc = (warps * sizeof(int4) + 255) & ~(size_t)255;
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
  const long long units = (long long)cache->batch * a.row_tiles * cache->n_kv_heads;
  long long tiles = ((long long)cache->max_pages * cache->page_tokens + 15) / 16;
  if (window > 0 && ((long long)window + n_q_tokens + 29) / 16 < tiles) tiles = ((long long)window + n_q_tokens + 29) / 16;
  a.cluster = ca_cluster_of(units, tiles, blocks);
  a.joins = !a.cluster && (long long)cache->max_pages * cache->page_tokens > 16 * CA_WHOLE;   // else no unit can have been cut
  DD_CUDA_TRY(nullptr, cudaFuncSetAttribute(p.main_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, p.smem_cluster));
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  dd_pdl_attr(&at[0]);
  cfg.attrs = at;
  cfg.numAttrs = 1;
  cfg.stream = (cudaStream_t)stream;
  cfg.blockDim = dim3(CA_THREADS);
  void* args[] = {&a};
  if (a.cluster) {
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)a.cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
    cfg.gridDim = dim3((unsigned)(units * a.cluster));
    cfg.dynamicSmemBytes = p.smem_cluster;
    return dd_launch(who, &cfg, p.main_kernel, args);
  }
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.dynamicSmemBytes = p.smem;
  DD_TRY(dd_launch(who, &cfg, p.main_kernel, args));
  if (!a.joins) return DD_OK;
  cfg.gridDim = dim3((unsigned)blocks, (unsigned)(nt * (cache->head_dim / 16) * 32 / 64));
  cfg.blockDim = dim3(64 * CJ_GROUPS);
  cfg.dynamicSmemBytes = (size_t)(blocks + 1) * 8 * sizeof(float);     // at most one partial per block and the last piece
  return dd_launch(who, &cfg, p.join_kernel, args);
}
