// The kernels of attention over a paged cache: of the newest tokens over all their tokens (dd_cache_attn.cu says how), and of query
// tokens over the pages listed for each (dd_cache_sparse.cu; SP = 1, and 2 for two tokens to a unit). 4-bit pages: see ca_scale4.
#pragma once

#include <type_traits>

#include "dd_cache.cuh"

namespace {

constexpr int CA_WARPS = 8;
constexpr int CA_THREADS = CA_WARPS * 32;
constexpr int CA_WHOLE = 8;                  // a unit of at most so many tiles is not cut: it belongs to the run it begins in
constexpr int CA_MAX_CLUSTER = 8;
constexpr float CA_LAZY = 8.f;               // how far (log2) a weight may exceed the reference
constexpr float CA_NONE = -3.0e38f;          // reference before any token: every finite score exceeds it

// formats: 0 bf16 pages and queries, 1 half pages and queries, 2 / 3 e4m3 pages with bf16 / half queries, 4 / 5 4-bit pages with the same
template <int FMT> struct ca_types { using Q = __nv_bfloat16; };
template <> struct ca_types<1> { using Q = __half; };
template <> struct ca_types<3> { using Q = __half; };
template <> struct ca_types<5> { using Q = __half; };
DD_HD constexpr bool ca_quantised(int fmt) { return fmt >= 2; }             // codes as halves, exponents of their own
DD_HD constexpr bool ca_int4(int fmt) { return fmt >= 4; }
constexpr float CA_INT4_BACK = 131072.f;                              // 4-bit values enter the products as 2^-17 of themselves
constexpr int CA_NOWHERE = 0x7ffffff0;                                // first token of a tile that is not there

template <int FMT, int D, int NT, int SP>
struct ca_geom {
  static constexpr bool FP8 = ca_quantised(FMT) && !ca_int4(FMT);
  static constexpr bool I4 = ca_int4(FMT);
  static constexpr int ES = FP8 ? 1 : 2;
  static constexpr int ROW = I4 ? D / 2 : D * ES;                     // bytes of a row: 64, 128 or 256 (4-bit: 32 or 64)
  static constexpr int HALF_BYTES = 16 * ROW;                         // K (or V) of a tile
  // What one copy group of a warp brings: K or V of a tile in turn, or a whole tile where that is small. Halves of 2 KiB keep
  // more in flight (e4m3 at head_dim 128, 8 x 32K tokens: 102 us against 108 with whole tiles), halves of 1 KiB cost more than they
  // bring (head_dim 64: 74 against 63 us), and with the deep ring of two column tiles whole tiles win (126 against 136 us).
  static constexpr bool WHOLE = I4 || 2 * HALF_BYTES <= (NT == 1 ? 2048 : 4096);
  static constexpr int EXP_AT = (WHOLE ? 2 : 1) * HALF_BYTES;         // e4m3: exponents of the tile, 16 of K and 16 of V, behind K or all
  static constexpr int TILE_BYTES = I4 ? dd_int4_tile_bytes(D) : (WHOLE ? 2 : 1) * HALF_BYTES + (FP8 ? 32 : 0);
  static constexpr int SLOT_BYTES = TILE_BYTES + (SP ? 16 : 0);       // listed pages: the tile's first token behind it
  static constexpr int COPIES = HALF_BYTES / 512;
  static constexpr int BLOCKS_PER_SM = NT == 1 ? 2 : 1;               // two column tiles need the registers of a whole SM
  static constexpr int RING_BUDGET = (BLOCKS_PER_SM == 2 ? 106 : 212) * 1024;
  static constexpr int STAGES_ = RING_BUDGET / (CA_WARPS * SLOT_BYTES);
  static constexpr int STAGES = STAGES_ > 8 ? 8 : STAGES_;
  // log2 of the factor on P: halves are lifted out of their subnormals; bf16 weights end at 1, so that large values do not
  // leave the range of the fp32 sums.
  static constexpr float HEADROOM = FMT == 0 ? -CA_LAZY : 6.f;
  // Weights as two 16-bit parts (see "Rounding").
  static constexpr bool PAIR = FMT != 2 && FMT != 4;
  // A second copy of the tile's code without masks and questions: 131 -> 111 us (128 query heads, 8 x 32K tokens e4m3), 63 -> 58
  // (head_dim 64), 106 -> 104 (e4m3, head_dim 128). bf16 and half pages with one column tile at head_dim 128 wait for memory with
  // either and go without; with listed pages, which mostly come from L2, they do not wait (2048 tokens of 64 pages: 591 -> 570 us).
  static constexpr bool PLAIN_LOOP = FP8 || I4 || NT == 2 || D == 64 || SP;
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

}  // namespace

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
  int batch;           // requests; of a call with listed pages: query tokens
  // listed pages (SP): every query token is a batch of its own, with a list of pages per KV head
  const int* positions;
  const int* requests; // NULL: tokens_per_request tokens of each in turn
  const int* idx;      // [batch][n_kv_heads][k_pages]
  int k_pages, tokens_per_request;
  int unit_tiles;      // tiles of a full list
  int unit_cost;       // empty places behind a unit in the flat list
  int n_tokens;
  // two tokens to a unit (Tq = 2, batch = pairs), where the lists of both have been made one: entries page | listed << 28 (bit 0: by the
  // first token, bit 1: by the second), -1 none; idx is [batch][n_kv_heads][k_pages] of them, and of a pair's entries so many are used
  const int* counts;
  int cluster;         // blocks of a cluster that share one unit, 0 = the flat list
  int joins;           // the joining kernel follows
  uint32_t by_G;       // ceil(2^31 / G): row / G by a multiplication
  float scale_log2;
};

namespace {

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
__device__ __forceinline__ float ca_max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
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

// Tokens [first, end) of a request that any of its query tokens sees, as tiles of 16. With listed pages: the token's position + 1
// in `end`, and the tiles of as many list entries as there are visible pages; none for a padding token or one that names no place.
struct ca_span {
  int end, first;      // tokens; first is the lowest visible one
  int tile0, tiles;
};
template <int SP> __device__ __forceinline__ ca_span ca_span_of(const ca_args& a, int b, bool report) {
  if constexpr (SP) {
    ca_span s = {0, 0, 0, 0};
    if constexpr (SP == 2) {                                          // what each token sees, its rows know
      s.end = 1;
      s.tiles = a.counts[b] << (a.c.page_shift - 4);
      return s;
    }
    const int pos = a.positions[b], req = a.requests ? a.requests[b] : b / a.tokens_per_request;
    if (pos < 0) return s;
    if ((unsigned)req >= (unsigned)a.c.batch || (pos >> a.c.page_shift) >= a.c.max_pages) {
      if (report) dd_status(a.c.status, (unsigned)req >= (unsigned)a.c.batch ? req : pos);
      return s;
    }
    s.end = pos + 1;
    s.tiles = min(a.unit_tiles, ((pos >> a.c.page_shift) + 1) << (a.c.page_shift - 4));
    return s;
  }
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

// Position of token `tok` of a pair, -1 where there is none.
__device__ __forceinline__ int ca_listed_position(const ca_args& a, long long tok) {
  if (tok >= a.n_tokens) return -1;
  const int pos = a.positions[tok], req = a.requests ? a.requests[tok] : (int)(tok / a.tokens_per_request);
  return pos >= 0 && (unsigned)req < (unsigned)a.c.batch && (pos >> a.c.page_shift) < a.c.max_pages ? pos : -1;
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
template <int SP> __device__ __forceinline__ void ca_next_unit(const ca_args& a, ca_cursor& k, int subs) {
  k.t = 0;
  if (++k.sub == subs) {
    k.sub = 0;
    do {
      if (k.b + 1 >= a.batch) { k.left = 0; return; }
      k.s = ca_span_of<SP>(a, ++k.b, false);
    } while (k.s.tiles == 0);
  }
  ca_keep_whole(k);
}
template <int SP> __device__ __forceinline__ void ca_step(const ca_args& a, ca_cursor& k, int subs) {
  --k.left;
  if (++k.t >= k.s.tiles) {
    k.left -= a.unit_cost;
    if (k.left > 0) ca_next_unit<SP>(a, k, subs);
  }
}

// Channel of accumulator m at row g of the product (row g + 8: the next one for quantised pages, else + 8).
template <int FMT, int D> __device__ __forceinline__ int ca_channel(int g, int m) {
  return ca_int4(FMT) ? g * (D / 8) + 2 * m : 16 * m + (ca_quantised(FMT) ? 2 * g : g);
}

// Two results of a query row (accumulator m, rows g and g + 8 of the product) to the row's output.
template <int FMT, int D> __device__ __forceinline__ void ca_store(char* row, int g, int m, uint32_t w) {
  char* at = row + 2 * ca_channel<FMT, D>(g, m);
  if (ca_quantised(FMT)) {
    *reinterpret_cast<uint32_t*>(at) = w;
  } else {
    *reinterpret_cast<unsigned short*>(at) = (unsigned short)w;
    *reinterpret_cast<unsigned short*>(at + 16) = (unsigned short)(w >> 16);
  }
}

// ---- 4-bit codes as halves. The four low nibbles of a half and the four of the other are the codes of four pairs; where a nibble lies
// it is a subnormal half, code * 2^-24 or code * 2^-20, so that one multiply-add gives (code - 8) * scale * 2^-17: exact for scales
// from 2^-4 on.
struct ca_scale4 { uint32_t at0, at4, off; };                         // half2: scale * 2^7, scale * 2^3, -scale * 2^-14
__device__ __forceinline__ uint32_t ca_hmul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t ca_hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
__device__ __forceinline__ ca_scale4 ca_scales4(uint32_t s) {         // of two scales as halves
  return {ca_hmul2(s, 0x58005800u), ca_hmul2(s, 0x48004800u), ca_hmul2(s, 0x84008400u)};
}
__device__ __forceinline__ uint32_t ca_e4m3x2_to_half(uint32_t codes) {
  uint32_t r;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\t}" : "=r"(r) : "r"(codes));
  return r;
}
__device__ __forceinline__ void ca_int4_pairs(uint32_t (&r)[4], uint32_t w, const ca_scale4& s) {
  const uint32_t hi = w >> 8;
  r[0] = ca_hfma2(w & 0x000f000fu, s.at0, s.off);
  r[1] = ca_hfma2(w & 0x00f000f0u, s.at4, s.off);
  r[2] = ca_hfma2(hi & 0x000f000fu, s.at0, s.off);
  r[3] = ca_hfma2(hi & 0x00f000f0u, s.at4, s.off);
}
__device__ __forceinline__ uint32_t ca_lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t ca_lds16(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a) : "memory");
  return v;
}
template <int N> __device__ __forceinline__ void ca_lds(uint32_t (&r)[N], uint32_t a) {
  if constexpr (N == 4)
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
  else
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(a) : "memory");
}
// x += v * (scale of the column): elements 0 and 2 belong to the lane's first column, 1 and 3 to its second
__device__ __forceinline__ void ca_add(float4& x, const float4& v, float s0, float s1) {
  x.x = fmaf(v.x, s0, x.x);
  x.y = fmaf(v.y, s1, x.y);
  x.z = fmaf(v.z, s0, x.z);
  x.w = fmaf(v.w, s1, x.w);
}

__device__ __forceinline__ float ca_lse(float from, float den) { return (from + log2f(den)) * 0.6931471805599453f; }

template <int FMT, int D, int NT, int SP>
__global__ void __launch_bounds__(CA_THREADS, (ca_geom<FMT, D, NT, SP>::BLOCKS_PER_SM)) dd_cache_attn_kernel(const ca_args a) {
  using geo = ca_geom<FMT, D, NT, SP>;
  constexpr bool PLAIN_LOOP = geo::PLAIN_LOOP;
  using TQ = typename ca_types<FMT>::Q;
  using TP = typename ca_types<FMT == 0 ? 0 : 1>::Q;
  constexpr bool FP8 = geo::FP8, I4 = geo::I4, QUANT = FP8 || I4;
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
  const int B = a.batch;
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
    is.s = ca_span_of<SP>(a, is.b, is.sub == 0 && w == 0);
    const int each = (is.s.tiles + a.cluster * CA_WARPS - 1) / (a.cluster * CA_WARPS);
    is.t = each * w;
    is.left = max(0, min(each, is.s.tiles - is.t));
  } else {
    // ---- this warp's run of the flat list
    auto places = [&](const ca_span& sp) -> long long { return sp.tiles > 0 ? (long long)(sp.tiles + a.unit_cost) * subs : 0; };
    long long cost0 = 0, total = 0;
    long long at = 0;                                                   // first place of the 32 requests looked at
    int from_b = 0;
    if constexpr (SP) {
      // query tokens may be many: every thread adds up an equal share of them, and the warp looks for its run in the share that has it
      long long* const sums = reinterpret_cast<long long*>(ca_smem);
      const int each = (B + CA_THREADS - 1) / CA_THREADS, b1 = min(B, ((int)threadIdx.x + 1) * each);
      for (int b = threadIdx.x * each; b < b1; ++b) total += places(ca_span_of<SP>(a, b, blockIdx.x == 0));
      long long incl = total;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      if (lane == 31) sums[CA_THREADS + warp] = incl;
      __syncthreads();
      long long before = 0;
      total = 0;
      for (int w = 0; w < CA_WARPS; ++w) {
        if (w < warp) before += sums[CA_THREADS + w];
        total += sums[CA_THREADS + w];
      }
      sums[threadIdx.x] = before + incl;                                // through this thread's share
      __syncthreads();
      share = max(1LL, ca_div(total + (long long)gridDim.x * CA_WARPS - 1, (int)gridDim.x * CA_WARPS));
      int in = 0;                                                       // the first share that reaches beyond f0
      for (int i = lane; i < CA_THREADS; i += 32) in += sums[i] <= share * me;
      in = (int)__reduce_add_sync(0xffffffffu, (unsigned)in);
      if (in > 0) at = sums[in - 1];
      from_b = in * each;
      __syncthreads();                                                  // the rings lie here
    } else {
      // every warp adds up the list by itself, 32 requests at a time
      is.s = ca_span_of<SP>(a, min(lane, B - 1), blockIdx.x == 0 && warp == 0 && lane < B);
      cost0 = lane < B ? places(is.s) : 0;                              // of the first 32 requests
      total = cost0;
      for (int b = lane + 32; b < B; b += 32) total += places(ca_span_of<SP>(a, b, blockIdx.x == 0 && warp == 0));
#pragma unroll
      for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    }
    share = max(1LL, ca_div(total + (long long)gridDim.x * CA_WARPS - 1, (int)gridDim.x * CA_WARPS));
    const long long f0 = share * me;
    if (f0 < total) {
      for (int b0 = from_b;; b0 += 32) {
        ca_span sp = is.s;
        long long cost = cost0;
        if (SP || b0 > 0) {
          sp = ca_span_of<SP>(a, min(b0 + lane, B - 1), false);
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
          is.sub = (int)ca_div(off, is.s.tiles + a.unit_cost);
          is.t = (int)(off - (long long)is.sub * (is.s.tiles + a.unit_cost));
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
        is.left -= is.s.tiles + a.unit_cost - is.t;
        if (is.left > 0) ca_next_unit<SP>(a, is, subs);
      }
    }
  }

  // ---- the issuing side
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ca_smem) + warp * geo::WARP_BYTES;
  ca_cursor u = is;                                  // the using side starts at the same place
  const int page_mask = (1 << a.c.page_shift) - 1;
  // Table entries of the next 32 tiles of the unit, one per lane.
  int blocks = 0, blocks_from = 0, blocks_of = -1;   // entries at hand, the first one's tile, their request
  int tokens = 0;                                    // listed pages: the first token of the lane's tile + who lists it, CA_NOWHERE = no such page
  const char* head_at = nullptr;                     // page 0 of the unit's head
  auto look_up = [&]() {
    blocks_from = is.t;
    blocks_of = is.b;
    const int i = min(is.t + lane, is.s.tiles - 1);
    if constexpr (SP) {
      const int per_page = a.c.page_shift - 4, rt = ca_row_tile(a, is.sub), head = is.sub - rt * a.c.n_kv_heads;
      int page = __ldg(a.idx + ((long long)is.b * a.c.n_kv_heads + head) * a.k_pages + (i >> per_page));
      blocks = 0;
      tokens = CA_NOWHERE;
      if constexpr (SP == 2) {
        if (page >= 0) {                                              // what is listed has been looked over
          const int listed = page >> 28, tok = 2 * is.b + (listed == 2);
          page &= 0xfffffff;
          const int req = a.requests ? __ldg(a.requests + tok) : tok / a.tokens_per_request;
          blocks = __ldg(a.c.table + req * a.c.table_stride + page);
          tokens = (page << a.c.page_shift) + ((i & ((1 << per_page) - 1)) << 4) + listed;
        }
        return;
      }
      const int req = a.requests ? __ldg(a.requests + is.b) : is.b / a.tokens_per_request;
      if (page < -1 || page >= a.c.max_pages) {
        dd_status(a.c.status, page);
      } else if (page >= 0 && page <= (is.s.end - 1) >> a.c.page_shift) {
        blocks = __ldg(a.c.table + req * a.c.table_stride + page);
        tokens = (page << a.c.page_shift) + ((i & ((1 << per_page) - 1)) << 4) + 1;
      }
      return;
    }
    blocks = __ldg(a.c.table + is.b * a.c.table_stride + (((is.s.tile0 + i) << 4) >> a.c.page_shift));
  };
  auto all_good = [&]() { return __all_sync(0xffffffffu, (unsigned)blocks < (unsigned)a.c.n_blocks); };
  auto enter_unit = [&]() {
    const int rt = ca_row_tile(a, is.sub), head = is.sub - rt * a.c.n_kv_heads;
    head_at = a.c.data + head * a.c.head_stride;
    // the next head of the same request has the same table: short units would wait for it anew at every head
    if (SP || blocks_of != is.b || blocks_from != 0 || is.t != 0) look_up();
    // The unit's query rows are called into L1 a few tiles ahead of their use, every 32-byte sector of them.
    constexpr int SECTORS = D / 16;
#pragma unroll
    for (int i = 0; i < NT * 8 * SECTORS; i += 32) {
      const int row = rt * NT * 8 + (i + lane) / SECTORS;
      if (row < a.n_rows && (SP != 2 || is.b * a.Tq + ca_token(a, row) < a.n_tokens)) {
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
    if constexpr (I4) {                              // a tile as it lies
      constexpr int N = geo::TILE_BYTES / 16;
#pragma unroll
      for (int i = 0; i < (N + 31) / 32; ++i)
        if (i * 32 + 32 <= N || i * 32 + lane < N) ca_cp16_all(to + (i * 32 + lane) * 16, from + (i * 32 + lane) * 16);
    } else {
#pragma unroll
      for (int i = 0; i < geo::COPIES; ++i)
        ca_cp16_all(to + (place0 ^ ca_twist<geo::ROW>(i)) + i * 512, from + i * 512 + lane * 16);
    }
  };
  auto copy_half = [&](uint32_t to, const char* from) {
    if constexpr (I4) {                              // the tokens that are not there are masked at their use
      if (n_valid > 0) {
        copy_full(to, from);
      } else {                                       // scales of zero: all zeros
        for (int i = lane; i < geo::TILE_BYTES / 16; i += 32) ca_cp16(to + i * 16, from, 0u);
      }
    } else if (n_first <= 0 && n_valid >= 16) {
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
        int tok0 = SP ? __shfl_sync(0xffffffffu, tokens, is.t - blocks_from) : (is.s.tile0 + is.t) << 4;
        int blk = __shfl_sync(0xffffffffu, blocks, is.t - blocks_from);
        if (SP && lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(put + geo::TILE_BYTES), "r"(tok0) : "memory");
        const int listed = tok0 & 15;
        if (SP) tok0 &= ~15;
        n_first = is.s.first - tok0;
        n_valid = SP == 2 ? (listed ? 16 : 0) : is.s.end - tok0;
        if ((unsigned)blk >= (unsigned)a.c.n_blocks) {
          if (lane == 0) dd_status(a.c.status, blk);
          blk = 0;
          n_valid = 0;                               // reads as zeros
        }
        const int in_page = tok0 & page_mask;
        const char* page = head_at + blk * a.c.block_stride;
        src = page + (I4 ? (in_page >> 4) * geo::TILE_BYTES : in_page * geo::ROW);
        copy_half(put, src);
        if (FP8 && lane < 8) {
          // exponents: K's behind all the codes of the page, V's behind those
          const char* ex = page + (2 * D + (lane >> 2)) * (page_mask + 1) + in_page + (lane & 3) * 4;
          ca_cp4(put + geo::EXP_AT + lane * 4, ex, n_valid > 0 ? 4u : 0u);
        }
      }
      if (geo::WHOLE || v_half) {
        if (!I4) copy_half(put + (geo::WHOLE ? geo::HALF_BYTES : 0), src + (page_mask + 1) * geo::ROW);
        ca_step<SP>(a, is, subs);
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
    const int tok0 = SP ? __shfl_sync(0xffffffffu, tokens, is.t - blocks_from) : (is.s.tile0 + is.t) << 4;
    const int in_page = tok0 & page_mask & ~15;
    if (SP && lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(put + geo::TILE_BYTES), "r"(tok0) : "memory");
    const char* page = head_at + __shfl_sync(0xffffffffu, blocks, is.t - blocks_from) * a.c.block_stride;
    src = page + (I4 ? (in_page >> 4) * geo::TILE_BYTES : in_page * geo::ROW);
    copy_full(put, src);
    if (FP8 && lane < 8) ca_cp4_all(put + geo::EXP_AT + lane * 4, page + (2 * D + (lane >> 2)) * (page_mask + 1) + in_page + (lane & 3) * 4);
    if (geo::WHOLE && !I4) copy_full(put + geo::HALF_BYTES, src + (page_mask + 1) * geo::ROW);
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
      if (row < a.n_rows && (SP != 2 || b * a.Tq + ca_token(a, row) < a.n_tokens)) {
        const int tok = ca_token(a, row);
        const char* qr = a.q + ((long long)b * a.Tq + tok) * a.q_token_stride + (head * a.G + row - tok * a.G) * a.q_head_stride;
        if constexpr (I4) {                                           // channels D/4 t ...: pairs (k, k + 4) of 8
#pragma unroll
          for (int w = 0; w < D / 32; ++w) {
            const uint4 v = *reinterpret_cast<const uint4*>(qr + 2 * (D / 4 * t + 8 * w));
            qf[nt][4 * w] = __byte_perm(v.x, v.z, 0x5410u);
            qf[nt][4 * w + 1] = __byte_perm(v.x, v.z, 0x7632u);
            qf[nt][4 * w + 2] = __byte_perm(v.y, v.w, 0x5410u);
            qf[nt][4 * w + 3] = __byte_perm(v.y, v.w, 0x7632u);
          }
        } else
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
      if (QUANT) {
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
        zs[nt][c] = a.scale_log2 * (QUANT ? __shfl_sync(0xffffffffu, back, (2 * t + c) * 4) * (I4 ? CA_INT4_BACK : 1.f) : 1.f);
        const int r = r0 + nt * 8 + 2 * t + c;
        pos[nt][c] = r < a.n_rows ? (SP == 2 ? ca_listed_position(a, 2LL * b + ca_token(a, r)) : s.end - a.Tq + ca_token(a, r)) : -1;
      }
    }
    int pos_lo = s.end - a.Tq + ca_token(a, r0);                             // positions of the first and last row of the tile
    int pos_hi = s.end - a.Tq + ca_token(a, min(a.n_rows, r0 + NT * 8) - 1);
    int everybody = 1;                                                // listed pages: the tokens there are, as bits
    if (SP == 2) {
      const int p0 = ca_listed_position(a, 2LL * b), p1 = ca_listed_position(a, 2LL * b + 1);
      pos_lo = p0 < 0 ? p1 : (p1 < 0 ? p0 : min(p0, p1));
      pos_hi = max(p0, p1);
      everybody = (p0 >= 0 ? 1 : 0) + (p1 >= 0 ? 2 : 0);
    }
    int who[NT][2];                                                   // pairs: the lane's columns' token, as a bit
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) who[nt][c] = SP == 2 ? 1 << min(ca_token(a, r0 + nt * 8 + 2 * t + c), 2) : 1;

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
    // ---- 4-bit tiles: scores (in two chains, without the scales of rows and queries), values' codes and scales, products with weights
    auto scores4 = [&](uint32_t slot, float (&z)[NT][4], float (&z2)[NT][4], float& by0, float& by1, float& vex0, float& vex1) {
      by0 = __uint_as_float(max((uint32_t)ca_lds_byte(slot + 18 * D + g) << 23, 0x00400000u));
      by1 = __uint_as_float(max((uint32_t)ca_lds_byte(slot + 18 * D + g + 8) << 23, 0x00400000u));
      vex0 = (float)(ca_lds_byte(slot + 18 * D + 16 + g) - 127);
      vex1 = (float)(ca_lds_byte(slot + 18 * D + 24 + g) - 127);
      uint32_t r0[D / 32], r1[D / 32];                                // rows g and g + 8: channels D/4 t ...
      ca_lds(r0, slot + lane * (D / 8));
      ca_lds(r1, slot + 4 * D + lane * (D / 8));
      // one scale for every 16 channels: two a lane (head_dim 128) or one
      constexpr int SC = D / 64;
      ca_scale4 m0[SC], m1[SC];
      if constexpr (D == 128) {
        const uint32_t s0 = ca_e4m3x2_to_half(ca_lds16(slot + 16 * D + g * 8 + t * 2)), s1 = ca_e4m3x2_to_half(ca_lds16(slot + 16 * D + 64 + g * 8 + t * 2));
        m0[0] = ca_scales4(__byte_perm(s0, 0u, 0x1010u));
        m0[1] = ca_scales4(__byte_perm(s0, 0u, 0x3232u));
        m1[0] = ca_scales4(__byte_perm(s1, 0u, 0x1010u));
        m1[1] = ca_scales4(__byte_perm(s1, 0u, 0x3232u));
      } else {
        m0[0] = ca_scales4(ca_e4m3x2_to_half((uint32_t)ca_lds_byte(slot + 16 * D + g * 4 + t) * 0x101u));
        m1[0] = ca_scales4(ca_e4m3x2_to_half((uint32_t)ca_lds_byte(slot + 16 * D + 32 + g * 4 + t) * 0x101u));
      }
#pragma unroll
      for (int w = 0; w < D / 32; ++w) {
        uint32_t h0[4], h1[4];
        ca_int4_pairs(h0, r0[w], m0[w / 2]);
        ca_int4_pairs(h1, r1[w], m1[w / 2]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          if (w == 0) {
            ca_mma_first<FMT>(z[nt], h0[0], h1[0], h0[1], h1[1], qf[nt][0], qf[nt][1]);
            ca_mma_first<FMT>(z2[nt], h0[2], h1[2], h0[3], h1[3], qf[nt][2], qf[nt][3]);
          } else {
            ca_mma<FMT>(z[nt], h0[0], h1[0], h0[1], h1[1], qf[nt][4 * w], qf[nt][4 * w + 1]);
            ca_mma<FMT>(z2[nt], h0[2], h1[2], h0[3], h1[3], qf[nt][4 * w + 2], qf[nt][4 * w + 3]);
          }
        }
      }
    };
    // tokens 2t, 2t + 1 | 2t + 8, 2t + 9, part g, and their scales
    auto values4 = [&](uint32_t slot, uint32_t (&v4)[2][D / 32], uint32_t (&vs4)[2]) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        ca_lds(v4[k], slot + 8 * D + (k * 32 + lane) * (D / 8));
        vs4[k] = ca_e4m3x2_to_half(ca_lds16(slot + 17 * D + (D == 128 ? g : g >> 1) * 16 + 8 * k + 2 * t));
      }
    };
    // one register of each token pair's codes in turn, dealt to the accumulators they feed: add(accumulator, fragment of V^T)
    auto weigh4 = [&](const uint32_t (&v4)[2][D / 32], const uint32_t (&vs4)[2], auto&& add) {
      const ca_scale4 m0 = ca_scales4(vs4[0]), m1 = ca_scales4(vs4[1]);
#pragma unroll
      for (int q = 0; q < D / 32; ++q) {                              // channels 4 q .. 4 q + 3 of the lane's part
        const uint32_t pick = (q & 1) ? 0x7632u : 0x5410u;
        uint32_t h0[4], h1[4];
        ca_int4_pairs(h0, __byte_perm(v4[0][q >> 1], v4[0][D / 64 + (q >> 1)], pick), m0);
        ca_int4_pairs(h1, __byte_perm(v4[1][q >> 1], v4[1][D / 64 + (q >> 1)], pick), m1);
        add(2 * q, h0[0], h0[1], h1[0], h1[1]);
        add(2 * q + 1, h0[2], h0[3], h1[2], h1[3]);
      }
    };
    // Two complete 4-bit tiles that every row sees at once: one question about the reference for both, and two chains of work that do not
    // wait for each other.
    auto pair4 = [&]() {
      constexpr int U = 2;
      constexpr float MOST = CA_LAZY + geo::HEADROOM;
      float z[U][NT][4], vex[U][2], by[U][2];                         // by: key scales
      uint32_t slot[U];
      ca_wait<NS - U>();
      __syncwarp();
      slot[0] = take;
      slot[1] = take + geo::SLOT_BYTES == ring + geo::WARP_BYTES ? ring : take + geo::SLOT_BYTES;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float z2[NT][4];
        scores4(slot[u], z[u], z2, by[u][0], by[u][1], vex[u][0], vex[u][1]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) z[u][nt][e] += z2[nt][e];
      }
      uint32_t pb[U][NT][2], pr[U][NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float x[U][4], y[U][4];
        float most = -INFINITY;                                       // of the weights' exponents, as if no value's scale were below 2^-96
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            z[u][nt][e] *= zs[nt][e & 1] * by[u][e >> 1];
            x[u][e] = z[u][nt][e] - from[nt][e & 1];
            y[u][e] = x[u][e] + vex[u][e >> 1];
          }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          most = ca_max3(most, x[u][0] + fmaxf(vex[u][0], -96.f), x[u][1] + fmaxf(vex[u][0], -96.f));
          most = ca_max3(most, x[u][2] + fmaxf(vex[u][1], -96.f), x[u][3] + fmaxf(vex[u][1], -96.f));
        }
        const bool above = most > MOST;
        if (__any_sync(0xffffffffu, above)) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float top = from[nt][c] + geo::HEADROOM;
#pragma unroll
            for (int u = 0; u < U; ++u) top = fmaxf(top, fmaxf(z[u][nt][c] + fmaxf(vex[u][0], -96.f), z[u][nt][2 + c] + fmaxf(vex[u][1], -96.f)));
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
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              x[u][e] = z[u][nt][e] - from[nt][e & 1];
              y[u][e] = x[u][e] + vex[u][e >> 1];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[e] = ca_exp2(y[u][e]);
            sum[nt][e & 1] += ca_exp2(x[u][e]);
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (geo::PAIR) {
              const uint32_t w = ca_first_part<TP>(p[2 * k], p[2 * k + 1]);
              const float2 had = dd_unpack2<TP>(w);
              pb[u][nt][k] = ca_transpose(w);
              pr[u][nt][k] = ca_transpose(dd_pack2<TP>(p[2 * k] - had.x, p[2 * k + 1] - had.y));
            } else {
              pb[u][nt][k] = ca_transpose(dd_pack2<TP>(p[2 * k], p[2 * k + 1]));
            }
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        uint32_t v4[2][D / 32], vs4[2];
        values4(slot[u], v4, vs4);
        use_up(true, true);
        weigh4(v4, vs4, [&](int m, uint32_t v0, uint32_t v1, uint32_t v2, uint32_t v3) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            ca_mma<FMT>(acc[nt][m], v0, v1, v2, v3, pb[u][nt][0], pb[u][nt][1]);
            if (geo::PAIR) ca_mma<FMT>(acc[nt][m], v0, v1, v2, v3, pr[u][nt][0], pr[u][nt][1]);
          }
        });
      }
    };
    auto tile = [&](auto plain_, int i) {
      constexpr bool plain = decltype(plain_)::value;                 // no mask, and the refills need no questions
      int tok0 = (first_tile + i) << 4;
      // ---- scores
      float z[NT][4];
      float vex0 = 0.f, vex1 = 0.f;                                   // log2 of the value scales of tokens g, g + 8
      ca_wait<NS - 1>();
      __syncwarp();
      int listed = 1;
      if (SP) {
        tok0 = (int)ca_lds32(take + geo::TILE_BYTES);
        if (SP == 2) listed = tok0 & 15;                              // (a single token lists all of its tiles)
        tok0 &= ~15;
      }
      {
        float z2[NT][4];                                              // two chains: the products of one depend on each other
        [[maybe_unused]] const uint32_t at = take + k_row;
        float by0 = 1.f, by1 = 1.f;                                   // key scales of tokens g, g + 8
        if constexpr (I4) {
          scores4(take, z, z2, by0, by1, vex0, vex1);
        } else if constexpr (FP8) {
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
          for (int e = 0; e < 4; ++e) z[nt][e] = (z[nt][e] + z2[nt][e]) * (QUANT ? zs[nt][e & 1] * (e < 2 ? by0 : by1) : zs[nt][e & 1]);
      }
      if (!geo::WHOLE) use_up(plain, true);
      // whole tiles: V is there already, its first registers come in behind the soft-max
      constexpr int V_LOADS = I4 ? 1 : D / (FP8 ? 32 : 16), V_BATCH = V_LOADS < 4 ? V_LOADS : 4;
      uint32_t raw[V_BATCH][4];
      auto load_values = [&](int c0) {
        const uint32_t at = take + v_row + (geo::WHOLE ? geo::HALF_BYTES : 0);
#pragma unroll
        for (int c = 0; c < V_BATCH; ++c) ca_ldsm_trans(raw[c], at + (v_x ^ ((c0 + c) << 5)));
      };
      [[maybe_unused]] uint32_t v4[2][D / 32], vs4[2] = {0u, 0u};
      if constexpr (I4) {
        values4(take, v4, vs4);
      } else if (geo::WHOLE) {
        load_values(0);
      }

      // ---- masks: z[.][0..1] is token tok0 + g, z[.][2..3] token tok0 + g + 8
      const bool partial = (SP || !plain) && ((SP == 2 && listed != everybody) || tok0 + 15 > pos_lo || (a.window > 0 && tok0 <= pos_hi - a.window));
      if (partial) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int tok = tok0 + g + (e < 2 ? 0 : 8), p = pos[nt][e & 1];
            if (tok > p || (a.window > 0 && tok <= p - a.window)) z[nt][e] = -INFINITY;
            if (SP == 2 && !(listed & who[nt][e & 1])) z[nt][e] = -INFINITY;
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
          y[e] = QUANT ? x[e] + (e < 2 ? vex0 : vex1) : x[e];
          above |= y[e] > CA_LAZY + geo::HEADROOM;
          if (QUANT) above |= x[e] > CA_LAZY + geo::HEADROOM + 96.f;
        }
        if (__any_sync(0xffffffffu, above)) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float top = QUANT ? fmaxf(z[nt][c] + fmaxf(vex0, -96.f), z[nt][2 + c] + fmaxf(vex1, -96.f)) : fmaxf(z[nt][c], z[nt][2 + c]);
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
            y[e] = QUANT ? x[e] + (e < 2 ? vex0 : vex1) : x[e];
          }
        }
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[e] = ca_exp2(y[e]);
          sum[nt][e & 1] += QUANT ? ca_exp2(x[e]) : p[e];
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
      if constexpr (I4) {
        if (!partial) {
          weigh4(v4, vs4, [&](int m, uint32_t v0, uint32_t v1, uint32_t v2, uint32_t v3) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              ca_mma<FMT>(acc[nt][m], v0, v1, v2, v3, pb[nt][0], pb[nt][1]);
              if (geo::PAIR) ca_mma<FMT>(acc[nt][m], v0, v1, v2, v3, pr[nt][0], pr[nt][1]);
            }
          });
        } else if (SP == 2 && tok0 + 15 <= pos_lo) {
          // one token of the pair lists the tile, and sees all of it: the other's columns take nothing
          weigh4(v4, vs4, [&](int m, uint32_t v0, uint32_t v1, uint32_t v2, uint32_t v3) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float one[4];
              ca_mma_first<FMT>(one, v0, v1, v2, v3, pb[nt][0], pb[nt][1]);
              if (geo::PAIR) ca_mma<FMT>(one, v0, v1, v2, v3, pr[nt][0], pr[nt][1]);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (listed & who[nt][e & 1]) acc[nt][m][e] += one[e];
            }
          });
        } else {
          // as below; a scale of zero makes a value zero
          const uint32_t had0 = vs4[0], had1 = vs4[1];
#pragma unroll 1
          for (int q = SP == 2 ? 0 : pos_lo; q <= (SP == 2 ? 1 : pos_hi); ++q) {
            const int p = SP == 2 ? ca_listed_position(a, 2LL * b + q) : q;
            if (SP == 2 && !(listed >> q & 1)) continue;
            uint32_t keep[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int tok = tok0 + 2 * t + 8 * k, first = a.window > 0 ? p - a.window : -1;
              keep[k] = ((tok <= p && tok > first) ? 0xffffu : 0u) | ((tok + 1 <= p && tok + 1 > first) ? 0xffff0000u : 0u);
            }
            vs4[0] = had0 & keep[0];
            vs4[1] = had1 & keep[1];
            weigh4(v4, vs4, [&](int m, uint32_t v0, uint32_t v1, uint32_t v2, uint32_t v3) {
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                float one[4] = {0.f, 0.f, 0.f, 0.f};
                ca_mma<FMT>(one, v0, v1, v2, v3, pb[nt][0], pb[nt][1]);
                if (geo::PAIR) ca_mma<FMT>(one, v0, v1, v2, v3, pr[nt][0], pr[nt][1]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (SP == 2 ? who[nt][e & 1] == 1 << q : pos[nt][e & 1] == p) acc[nt][m][e] += one[e];
              }
            });
          }
        }
      } else if (!(partial && a.Tq > 1)) {
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
      } else if (SP == 2 && tok0 + 15 <= pos_lo) {
        // one token of the pair lists the tile, and sees all of it: the other's columns take nothing
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
                float one[4];
                ca_mma_first<FMT>(one, r[0], r[1], r[2], r[3], pb[nt][0], pb[nt][1]);
                if (geo::PAIR) ca_mma<FMT>(one, r[0], r[1], r[2], r[3], pr[nt][0], pr[nt][1]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (listed & who[nt][e & 1]) acc[nt][FP8 ? 2 * (c0 + c) + half : c0 + c][e] += one[e];
              }
            }
        }
      } else {
        // Some tokens are seen by some rows of the tile and not by others: a weight of zero does not keep an infinity or NaN
        // of V out of the sum, so the products are taken query token by query token with the unseen values made zero.
#pragma unroll 1
        for (int q = SP == 2 ? 0 : pos_lo; q <= (SP == 2 ? 1 : pos_hi); ++q) {
          const int p = SP == 2 ? ca_listed_position(a, 2LL * b + q) : q;
          if (SP == 2 && !(listed >> q & 1)) continue;
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
                    if (SP == 2 ? who[nt][e & 1] == 1 << q : pos[nt][e & 1] == p) acc[nt][FP8 ? 2 * (c0 + c) + half : c0 + c][e] += one[e];
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
      if (SP && PLAIN_LOOP && is.left > 1) {
        // tiles of the lookup from here on that are there, complete and visible; not the last of the run, of the unit or of the lookup.
        // Where V of a tile goes with K of the next, the next has to be one too.
        const unsigned odd = __ballot_sync(0xffffffffu, (SP == 2 ? tokens == CA_NOWHERE : (tokens & ~15) > is.s.end - 16) || (unsigned)blocks >= (unsigned)a.c.n_blocks) >> (is.t - blocks_from);
        n = (odd ? __ffs(odd) - 1 : 32 - (is.t - blocks_from)) - (V_FIRST ? 1 : 0);
        n = min(min(n, is.left - 1), min(blocks_from + 31 - is.t, is.s.tiles - 1 - is.t));
        n = min(n, n_here - i);
      } else if (PLAIN_LOOP && is.left > 1) {
        n = min(min(is.left, blocks_from + 32 - is.t), ((is.s.end - 16) >> 4) - is.s.tile0 - is.t + 1) - 1;
        n = min(n, min(n_here - i, ((pos_lo - 15) >> 4) - (first_tile + i) + 1));
        if (a.window > 0 && (((first_tile + i) << 4) <= pos_hi - a.window || ((is.s.tile0 + is.t) << 4) < is.s.first)) n = 0;
        if (!all_good()) n = 0;
      }
      if constexpr (I4) {
#pragma unroll 1
        for (; n > 1; n -= 2, i += 2) {
          if (SP) {                                                   // nobody has looked where the tiles to be used lie
            const uint32_t next = take + geo::SLOT_BYTES == ring + geo::WARP_BYTES ? ring : take + geo::SLOT_BYTES;
            const int at0 = (int)ca_lds32(take + geo::TILE_BYTES), at1 = (int)ca_lds32(next + geo::TILE_BYTES);
            if ((max(at0, at1) & ~15) > pos_lo - 15 || (SP == 2 && ((at0 & 15) != everybody || (at1 & 15) != everybody))) break;
          }
          pair4();
        }
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
    if (I4) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int m = 0; m < D / 16; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[nt][m][e] *= CA_INT4_BACK;
    }
    const bool ends = t0 + n_here == s.tiles;
    if (a.cluster) break;                                             // one piece a warp
    if (ends && t0 == 0) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int r = r0 + nt * 8 + 2 * t + c;
          if (r < a.n_rows && (SP != 2 || pos[nt][c] >= 0)) {
            const int tok = ca_token(a, r), h = head * a.G + r - tok * a.G;
            const long long tn = (long long)b * a.Tq + tok;
            const bool empty = SP ? sum[nt][c] == 0.f : pos[nt][c] < 0;   // (nothing listed, or before the beginning)
            const float inv = empty ? 0.f : __frcp_rn(sum[nt][c]);
            char* o = a.out + tn * a.out_token_stride + h * a.out_head_stride;
#pragma unroll
            for (int m = 0; m < D / 16; ++m) ca_store<FMT, D>(o, g, m, empty ? 0u : dd_pack2<TQ>(acc[nt][m][c] * inv, acc[nt][m][2 + c] * inv));
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
    u.left -= n_here + a.unit_cost;
    if (u.left > 0) ca_next_unit<SP>(a, u, subs);
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
  // units without a token: zeros and -inf, shared out over the blocks (listed pages: padding, whose rows stay as they are)
  for (int b = blockIdx.x; b < B && !SP; b += gridDim.x) {
    if (ca_span_of<SP>(a, b, false).tiles == 0) {
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
      const ca_span s = ca_span_of<SP>(a, b, false);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int r = rt * NT * 8 + row + c;
        if (r < a.n_rows && s.tiles > 0) {           // (a request without a token has been written above)
          const int tok = ca_token(a, r), h = head * a.G + r - tok * a.G;
          const long long tn = (long long)b * a.Tq + tok;
          const bool empty = SP ? L[c] == 0.f : s.end - a.Tq + tok < 0;
          const float lo = c ? x.y : x.x, hi = c ? x.w : x.z;
          ca_store<FMT, D>(a.out + tn * a.out_token_stride + h * a.out_head_stride, ge, m, empty ? 0u : dd_pack2<TQ>(lo / L[c], hi / L[c]));
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
template <int FMT, int D, int NT, int SP>
__global__ void __launch_bounds__(64 * CJ_GROUPS) dd_cache_attn_join_kernel(const ca_args a) {
  using TQ = typename ca_types<FMT>::Q;
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
    const int end = ca_span_of<SP>(a, b, false).end;
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
      if (r < a.n_rows && (SP != 2 || ca_listed_position(a, 2LL * b + ca_token(a, r)) >= 0)) {
        const int tok = ca_token(a, r), h = head * a.G + r - tok * a.G;
        const long long tn = (long long)b * a.Tq + tok;
        const float2 ml = sh_ml[col + c];
        const bool empty = SP ? ml.y == 0.f : end - a.Tq + tok < 0;
        ca_store<FMT, D>(a.out + tn * a.out_token_stride + h * a.out_head_stride, ge, m, empty ? 0u : dd_pack2<TQ>(lo / ml.y, hi / ml.y));
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
template <int FMT, int D, int NT, int SP> ca_plan ca_plan_of() {
  using geo = ca_geom<FMT, D, NT, SP>;
  static_assert(geo::SMEM_CLUSTER + 2048 <= 227 * 1024, "shared memory of a block");
  static_assert(geo::BLOCKS_PER_SM == 1 || geo::SMEM_CLUSTER + 1024 + 2048 <= 114 * 1024, "shared memory of two blocks");
  return {(const void*)dd_cache_attn_kernel<FMT, D, NT, SP>, (const void*)dd_cache_attn_join_kernel<FMT, D, NT, SP>, geo::SMEM, geo::SMEM_CLUSTER, geo::BLOCKS_PER_SM};
}
template <int FMT, int SP> ca_plan ca_pick_of(int d, int nt) {
  if constexpr (SP == 2) return d == 128 ? ca_plan_of<FMT, 128, 1, SP>() : ca_plan_of<FMT, 64, 1, SP>();      // up to 8 rows
  if (d == 128) return nt == 1 ? ca_plan_of<FMT, 128, 1, SP>() : ca_plan_of<FMT, 128, 2, SP>();
  return nt == 1 ? ca_plan_of<FMT, 64, 1, SP>() : ca_plan_of<FMT, 64, 2, SP>();
}

inline int ca_sm_count() {
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
inline int ca_cluster_of(long long units, long long tiles, int blocks) {
  if (tiles <= CA_WHOLE) return 0;
  int c = 2;
  while (c < CA_MAX_CLUSTER && tiles > 2LL * c * CA_WARPS) c *= 2;
  return tiles <= 8LL * c * CA_WARPS && units * c <= blocks * 7 / 8 ? c : 0;
}

// Rows of a unit that go through the MMA together: up to 8 in one column tile, up to 16 in two.
inline int ca_column_tiles(int rows) { return rows <= 8 ? 1 : 2; }

// The same for 4-bit pages and for listed pages, whose tiles take longer to work on than to bring: short units too go to the warps of a block
// (a cluster of one: 7 tiles one after the other in one warp 11.7 us, 7.9 side by side), and clusters as large as all units leave
// room for, up to two tiles a warp.
inline int ca_cluster_spread(long long units, long long tiles, int blocks) {
  int c = 1;
  while (c < CA_MAX_CLUSTER && tiles > 2LL * c * CA_WARPS) c *= 2;
  while (c > 1 && units * c > blocks * 7 / 8) c /= 2;
  return tiles > 1 && tiles <= 8LL * c * CA_WARPS && units * c <= blocks * 7 / 8 ? c : 0;
}

template <int SP> ca_plan ca_pick(int format, int d, int nt) {
  switch (format) {
    case 0: return ca_pick_of<0, SP>(d, nt);
    case 1: return ca_pick_of<1, SP>(d, nt);
    case 2: return ca_pick_of<2, SP>(d, nt);
    case 3: return ca_pick_of<3, SP>(d, nt);
    case 4: return ca_pick_of<4, SP>(d, nt);
    default: return ca_pick_of<5, SP>(d, nt);
  }
}

// Empty places behind a unit, for what it costs besides its tiles, by measurement (us with 3 | 5 | 8 places). 4-bit pages: 48 requests of 0 to 32K
// tokens 68 | 60.2 | 59.5 (12: 61.5), at head_dim 64 49.7 | 43.2 | 40.1, 100 requests of up to 5000 47.6 | 46.4 | 46.1. Listed pages, 481 ragged
// tokens at head_dim 64: e4m3 41.8 | 38.2 | 40.5, half 41.7 | 37.7 | 40.7, 4 bits 42.8 | 40.2 | 40.3; 450 at head_dim 128, a group of five: bf16
// 137.0 | 137.8 | 147.3, e4m3 119.7 | 120.1 | 120.3, 4 bits 134.6 | 124.5 | 122.6.
inline int ca_unit_cost(int cache_format, bool listed) { return cache_format == DD_CACHE_INT4 ? 8 : (listed ? 5 : 3); }

// Kernel format of a cache's pages and a type of queries.
inline int ca_format(int cache_format, int dtype) {
  const int half = dtype == DD_FP16;
  return cache_format == DD_CACHE_E4M3 ? 2 + half : (cache_format == DD_CACHE_INT4 ? 4 + half : half);
}

// The attention kernel and, where units may be cut, the joining one.
inline int ca_launch(const char* who, ca_args& a, const ca_plan& p, long long units, int blocks, int nt, int head_dim, cudaStream_t stream) {
  DD_TRY(dd_allow_smem(who, p.main_kernel, p.smem_cluster));
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  dd_pdl_attr(&at[0]);
  cfg.attrs = at;
  cfg.numAttrs = 1;
  cfg.stream = stream;
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
  cfg.gridDim = dim3((unsigned)blocks, (unsigned)(nt * (head_dim / 16) * 32 / 64));
  cfg.blockDim = dim3(64 * CJ_GROUPS);
  cfg.dynamicSmemBytes = (size_t)(blocks + 1) * 8 * sizeof(float);     // at most one partial per block and the last piece
  return dd_launch(who, &cfg, p.join_kernel, args);
}

struct ca_sizes { size_t part_o, part_ml, desc; size_t total() const { return part_o + part_ml + desc; } };
inline ca_sizes ca_size(int head_dim, int rows, int sms) {
  const int nt = ca_column_tiles(rows);
  const size_t warps = (size_t)sms * (nt == 1 ? 2 : 1) * CA_WARPS;
  ca_sizes z;
  z.part_o = 2 * warps * nt * 8 * head_dim * sizeof(float);
  z.part_ml = 2 * warps * nt * 8 * sizeof(float2);
  z.desc = (warps * sizeof(int4) + 255) & ~(size_t)255;
  return z;
}

inline const char* ca_check_heads(int n_q_heads, int n_kv_heads, int head_dim, int n_q_tokens) {
  if (head_dim != 64 && head_dim != 128) return "head_dim must be 64 or 128";
  if (n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads) return "n_q_heads must be a multiple of n_kv_heads";
  if (n_q_tokens < 1 || n_q_tokens > 64) return "n_q_tokens must be in [1, 64]";
  if (n_q_heads / n_kv_heads > 1024) return "more than 1024 query heads per KV head";
  return nullptr;
}

}  // namespace
