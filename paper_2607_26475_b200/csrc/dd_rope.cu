// Rotary positions and the writing of the paged key-value cache: one kernel for both, since a new token's keys are turned
// and stored in the same pass.
//
// A pair (u, w) of a row at position p is turned by the angle a = 2 pi p f (f turns per position):
//   u' = A (u cos a - w sin a),  w' = A (w cos a + u sin a)
// The angle is what loses precision: p f has to be known modulo 1 to a fraction of 2^-24 while p reaches millions, so the
// product and its reduction are done in 64 bits (two operations a pair and token, shared by all heads of the token); the
// remainder, at most half a turn, is split into an fp32 value and a correction of first order.
//
// Bound: HBM. Every row is read once and written once; there is no reuse. A group of head_dim / 16 lanes owns one token
// and a slice of its heads; each lane keeps the two 16-byte chunks of a row whose elements turn with each other (half
// layout: chunk j and chunk j + rot_dim / 16; interleaved: neighbours), so the rotation needs no exchange between lanes,
// and the sines and cosines of its eight pairs stay in registers for all heads of the slice. A quantised row's largest
// magnitude is one reduction over the group. 80 registers (one kind of rows at a time) keep three blocks on an SM; 4-bit rows take 128
// and two blocks.
//
// Measured on a B200: 32768 tokens of 32 + 8 heads of 128 bf16, rotation 102.5 us (6.55 TB/s, a copy's rate); the same with
// 8 + 8 heads of K and V into e4m3 pages 120 us (6.2 TB/s); into 4-bit pages 163 us (4.35 TB/s): 108 us of bytes and 65 us of
// issue slots, one after the other, since 14 warps an SM wait for a batch of rows and then work on it; 8 tokens 2.1 us (4-bit 3.6), one launch.
#include <math.h>

#include <type_traits>

#include "dd_cache.cuh"

namespace {

constexpr int RP_THREADS = 256;
constexpr int rp_blocks(int fmt) { return fmt == DD_CACHE_INT4 ? 2 : 3; }      // per SM, by registers
constexpr int RP_BATCH = 4;          // heads whose loads are in flight together

struct rp_rows {
  char* data;
  long long token_stride, head_stride;   // bytes
};

struct rp_args {
  const double* turns;
  const int* positions;
  const int* requests;
  rp_rows q, k, v, q_out, k_out;
  int n_tokens, n_q, n_k;            // n_k: heads of k and (append) of v
  int rot16;                         // rot_dim / 16, 0 = nothing is turned
  int interleaved, backward;
  float amplitude;
  int tokens_per_request;            // used when requests is NULL
  int slices, slice_heads;
  dd_cache_view cache;
};

__device__ __forceinline__ void rp_angle(double turns, int pos, float amplitude, float& c, float& s) {
  double a = turns * (double)pos;
  a -= rint(a);
  const float hi = (float)a;
  const float lo = (float)(a - (double)hi) * 6.283185307179586f;
  float s0, c0;
  sincospif(2.f * hi, &s0, &c0);
  c = fmaf(-s0, lo, c0) * amplitude;
  s = fmaf(c0, lo, s0) * amplitude;
}

// ---- 4-bit rows
// A row is 2^e times groups of 16 whole numbers times their group's scale. A lane holds two chunks of 8 elements; the other half of a
// chunk's group may lie with another lane (rp_mate). What is done for each element is kept to five instructions:
//   values as they came: q = x / (scale 2^e) by the inverse and one correction, exact where the quotient can be represented, so that ties
//     fall as in the definition; q + 1.5 2^23 + 8 has the code in its lowest bits; a shift and add per element collects the word (the
//     constant parts of all eight come off at the end). A quotient is at most 7 * 17 / 16 < 7.5, so no code is cut off.
//   turned values: known in 32 bits to 2^-21.2 of their pair's magnitude (sine and cosine 2^-22 each, product and sum), that is to
//     RP_KNOWN of the row's largest. Where that leaves a border within reach of the row's exponent, of a scale or of a code (a
//     few elements in 100,000), it is done again in 64 bits, the element or the row, so that the bytes written are those of the 64-bit
//     rotation (without a correction otherwise).
// Rows below 2^-108, rows that are not finite and rows turned with an amplitude below 2^-100 take the same 64-bit way; a turned element
// beyond what 32 bits hold counts as infinite, so that a row's exponent always fits its byte. Rows of zeros need no decision (what 32 bits
// make zero is far below half a code): 32768 tokens of zeros 154 us, 792 in 64 bits.
constexpr float RP_KNOWN = 0x1.8p-21f;
constexpr float RP_LEAST = 0x1p-100f;                  // amplitudes below it: sines and cosines times it may lose bits to subnormals
constexpr double RP_MOST = 0x1.fffffep127;             // the largest 32-bit number
constexpr unsigned RP_NEAR_MOST = 0x7f7fffe0u;         // bits of 2^128 less 2^-19 of it: further from RP_MOST than RP_KNOWN reaches

// Lane of the group and slot (0 or 1) that hold chunk `chunk` of a row.
__device__ __forceinline__ void rp_mate(int chunk, int rot16, bool interleaved, int& lane, int& slot) {
  if (interleaved || chunk >= 2 * rot16) {
    lane = chunk >> 1;
    slot = chunk & 1;
  } else {
    slot = chunk >= rot16;
    lane = chunk - slot * rot16;
  }
}

// Is s, known to eps, within reach of a point where its rounding to 4 significant bits changes?
__device__ __forceinline__ bool rp_near_scale(float s, float eps) {
  const int rest = (int)(__float_as_uint(s) & 0xfffffu) - 0x80000;
  return fabsf((float)rest) * (__uint_as_float(__float_as_uint(s) & 0x7f800000u) * 0x1p-23f) <= eps;
}
__device__ __forceinline__ float rp_round_e4m3(float v, unsigned& code) {
  code = dd_float_to_e4m3x4(v, v, 0.f, 0.f) & 0xffu;
  uint32_t h, unused;
  dd_e4m3x4_to_half(code, h, unused);
  return dd_unpack2<__half>(h).x;
}
__device__ __forceinline__ float rp_rcp(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// a / 7, exact where it can be represented.
__device__ __forceinline__ float rp_seventh(float a) {
  const float q = a * 0.14285714924335479736328125f;
  return fmaf(fmaf(-7.f, q, a), 0.14285714924335479736328125f, q);
}

// Where a lane's two chunks are and where the other chunk of each one's group is: lane (of the warp) and slot.
struct rp_place {
  int c0, c1, mate0, mate1, slots;
};

// One row in 64 bits, from its source: exponent byte (returned), scales (as e4m3 codes) and codes of the lane's two chunks.
template <typename T, int D>
__device__ __noinline__ int rp_int4_slow(const char* row, rp_place at, const double* turns, int pos, float amplitude, int j, bool interleaved,
                                         unsigned peers, unsigned (&scale)[2], uint32_t (&code)[2]) {
  double x[16], top[2] = {0., 0.};
  bool bad[2] = {false, false};
  for (int i = 0; i < 16; ++i) x[i] = (double)dd_to_float(reinterpret_cast<const T*>(row)[(i < 8 ? at.c0 : at.c1 - 8) + i]);
  for (int i = 0; turns && i < 8; ++i) {
    double a = turns[8 * j + i] * (double)pos, sn, cs;
    a -= rint(a);
    sincospi(2. * a, &sn, &cs);
    sn *= (double)amplitude;
    cs *= (double)amplitude;
    const int iu = interleaved ? 2 * i : i, iw = interleaved ? 2 * i + 1 : 8 + i;
    const double u = x[iu], w = x[iw];
    x[iu] = u * cs - w * sn;
    x[iw] = w * cs + u * sn;
  }
  for (int i = 0; i < 16; ++i) {
    const double m = fabs(x[i]);
    if (m <= RP_MOST) top[i >> 3] = fmax(top[i >> 3], m);
    else bad[i >> 3] = true;
  }
  double amax = fmax(top[0], top[1]);
  for (int m = 1; m < D / 16; m <<= 1) amax = fmax(amax, __shfl_xor_sync(peers, amax, m));
  int e = -127;
  if (amax > 0.) {
    e = ilogb(amax) - 11;
    if (amax > ldexp(3136., e)) ++e;
    e = max(e, -127);
  }
  for (int c = 0; c < 2; ++c) {
    const int mate = c ? at.mate1 : at.mate0, slot = (at.slots >> c) & 1;
    const double t0 = __shfl_sync(peers, top[0], mate), t1 = __shfl_sync(peers, top[1], mate);
    const int b = __shfl_sync(peers, (int)bad[0] + 2 * (int)bad[1], mate);
    const double r = fmax(ldexp(fmax(top[c], slot ? t1 : t0), -e) / 7., 0x1p-4);
    const double unit = ldexp(1., ilogb(r) - 3);
    const double s = rint(r / unit) * unit;                    // at most 448: four significant bits, an e4m3 value
    (void)rp_round_e4m3((float)s, scale[c]);
    const bool none = bad[c] || ((b >> slot) & 1);
    if (none) scale[c] = 0x7fu;
    uint32_t w = 0;
    for (int i = 0; i < 8; ++i) {
      const double n = none ? 0. : fmin(fmax(rint(ldexp(x[8 * c + i], -e) / s), -7.), 7.);
      w |= (uint32_t)((int)n + 8) << (4 * i);
    }
    code[c] = w;
  }
  return e + 127;
}

// The code of element e (0 .. 15) of a lane's chunks of a turned row (turns NULL: of a part that is not turned), in 64 bits, for an exponent byte and a scale that are certain.
template <typename T>
__device__ __noinline__ uint32_t rp_int4_element(const char* row, int c0, int c1, int e, const double* turns, int pos, float amplitude, int j,
                                                 bool interleaved, int byte, unsigned scale) {
  const int i = interleaved ? e >> 1 : e & 7, iu = interleaved ? 2 * i : i, iw = interleaved ? 2 * i + 1 : 8 + i;
  auto at = [&](int k) { return (double)dd_to_float(reinterpret_cast<const T*>(row)[k < 8 ? c0 + k : c1 + k - 8]); };
  double x = at(e);
  if (turns) {
    double a = turns[8 * j + i] * (double)pos, sn, cs;
    a -= rint(a);
    sincospi(2. * a, &sn, &cs);
    const double u = at(iu), w = at(iw);
    x = (e == iu ? u * cs - w * sn : w * cs + u * sn) * (double)amplitude;
  }
  uint32_t h, unused;
  dd_e4m3x4_to_half(scale, h, unused);
  const double n = rint(x * __hiloint2double((1023 + 127 - byte) << 20, 0) / (double)dd_unpack2<__half>(h).x);
  return (uint32_t)((int)fmin(fmax(n, -7.), 7.) + 8);
}

// FMT: -1 rotation only; DD_CACHE_* append. T: type of the rows.
template <typename T, int D, int FMT>
__global__ void __launch_bounds__(RP_THREADS, rp_blocks(FMT)) dd_rope_kernel(rp_args a) {
  constexpr int LANES = D / 16;
  constexpr int PER_WARP = 32 / LANES;
  const int lane = threadIdx.x & 31, j = lane % LANES;
  const unsigned peers = LANES == 8 ? 0xffu << (lane & 24) : 0xfu << (lane & 28);      // the lanes that share a token
  const int n_heads = a.n_q + a.n_k * (FMT >= 0 ? 2 : 1);
  // A block holds neighbouring tokens of one slice of the heads, and neighbouring blocks the slices of the same tokens, so that kinds of
  // rows that keep memory busy and kinds that keep the cores busy run side by side (32768 tokens: rotation 108 -> 102 us, e4m3 append
  // 134 -> 127; slices mixed within a block make it wait for its slowest warp: 4-bit append 189 -> 311 us).
  const unsigned over = blockIdx.x / (unsigned)a.slices;
  const int slice = blockIdx.x - over * a.slices;
  const long long n_ = ((long long)over * (RP_THREADS / 32) + (threadIdx.x >> 5)) * PER_WARP + lane / LANES;
  if (n_ - lane / LANES >= a.n_tokens) return;                 // a whole warp
  const int h0 = slice * a.slice_heads, h1 = min(n_heads, h0 + a.slice_heads);

  dd_grid_dependency_wait();
  const bool inside = n_ < a.n_tokens;
  const long long n = inside ? n_ : 0;
  const int pos = a.positions[n];
  bool live = inside && pos >= 0;

  char* page_at = nullptr;                                     // the token's page of KV head 0, and its place in it
  int off = 0;
  const int page_tokens = FMT >= 0 ? 1 << a.cache.page_shift : 0;
  if (FMT >= 0 && live) {
    const int req = a.requests ? a.requests[n] : (int)(n / a.tokens_per_request);
    const int pg = pos >> a.cache.page_shift;
    off = pos & (page_tokens - 1);
    if (req < 0 || req >= a.cache.batch) {
      dd_status(a.cache.status, req);
      live = false;
    } else if (pg >= a.cache.max_pages) {
      dd_status(a.cache.status, pg);
      live = false;
    } else {
      const int blk = a.cache.table[req * a.cache.table_stride + pg];
      if (blk < 0 || blk >= a.cache.n_blocks) {
        dd_status(a.cache.status, blk);
        live = false;
      } else {
        page_at = a.cache.data + blk * a.cache.block_stride;
      }
    }
  }

  const bool turned = j < a.rot16;
  float cs[8], sn[8];
  if (turned && (FMT < 0 || h0 < a.n_q + a.n_k)) {             // a slice of values alone needs no angles
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      rp_angle(a.turns[8 * j + i], pos, a.amplitude, cs[i], sn[i]);
      if (a.backward) sn[i] = -sn[i];
    }
  }
  // the two chunks of a row this lane owns (elements)
  int c0, c1;
  if (a.interleaved) { c0 = 16 * j; c1 = c0 + 8; }
  else if (turned) { c0 = 8 * j; c1 = c0 + 8 * a.rot16; }
  else { c0 = 16 * a.rot16 + 16 * (j - a.rot16); c1 = c0 + 8; }
  // 4-bit rows: where the other chunk of each chunk's group is; values are not turned and lie two neighbouring chunks to a lane
  rp_place place = {c0, c1, 0, 0, 0};
  bool same_lane = true, next_lane = false;
  if (FMT == DD_CACHE_INT4) {
    int slot0, slot1;
    rp_mate((c0 >> 3) ^ 1, a.rot16, a.interleaved, place.mate0, slot0);
    rp_mate((c1 >> 3) ^ 1, a.rot16, a.interleaved, place.mate1, slot1);
    place.mate0 += lane - j;
    place.mate1 += lane - j;
    place.slots = slot0 + 2 * slot1;
    same_lane = c1 == c0 + 8 && !(c0 & 8);
    next_lane = a.interleaved || a.rot16 % 2 == 0;             // the same for all lanes: no group reaches further than the next lane
  }
  const rp_place plain_place = {16 * j, 16 * j + 8, lane, lane, 1};

  // One kind of rows at a time (0 queries, 1 keys, 2 values), heads [lo, hi) of it.
  auto rows = [&](auto kind_, int lo, int hi, const rp_rows& from, const rp_rows& to) {
    constexpr int kind = decltype(kind_)::value;
    constexpr bool paged = FMT >= 0 && kind > 0;               // goes to the cache
    if (lo >= hi) return;
    const char* in = from.data + n * from.token_stride + lo * from.head_stride;
    char* out = nullptr;
    long long out_stride;
    if (paged) {
      out_stride = a.cache.head_stride;
      if (live) out = page_at + lo * out_stride;
    } else {
      out_stride = to.head_stride;
      out = to.data + n * to.token_stride + lo * out_stride;
    }
    constexpr bool quantised = paged && (FMT == DD_CACHE_E4M3 || FMT == DD_CACHE_INT4);
    const int row_off = paged ? ((kind == 2 ? page_tokens : 0) + off) * (FMT == DD_CACHE_E4M3 ? D : 2 * D) : 0;
    [[maybe_unused]] auto put4 = [&](char* page, const unsigned (&scale)[2], const uint32_t (&code)[2], int byte) {
      const int t = off & 15;
      char* tile = page + (off >> 4) * dd_int4_tile_bytes(D);
      if (kind == 2) {                                         // both chunks of a group
        if (D == 128) {
          *reinterpret_cast<uint2*>(tile + dd_int4_v_at<D>(t, 2 * j)) = make_uint2(code[0], code[1]);
        } else {
          *reinterpret_cast<uint32_t*>(tile + dd_int4_v_at<D>(t, 2 * j)) = code[0];
          *reinterpret_cast<uint32_t*>(tile + dd_int4_v_at<D>(t, 2 * j + 1)) = code[1];
        }
        tile[dd_int4_vs_at<D>(t, j)] = (char)scale[0];
      } else {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int chunk = (c ? c1 : c0) >> 3;
          *reinterpret_cast<uint32_t*>(tile + dd_int4_k_at<D>(t, chunk)) = code[c];
          if (!(chunk & 1)) tile[dd_int4_ks_at<D>(t, chunk >> 1)] = (char)scale[c];
        }
      }
      if (j == 0) tile[18 * D + (kind == 2 ? 16 : 0) + t] = (char)byte;
    };
    const int e0 = FMT == DD_CACHE_INT4 && kind == 2 ? 16 * j : c0, e1 = FMT == DD_CACHE_INT4 && kind == 2 ? 16 * j + 8 : c1;
    for (int h = lo; h < hi; h += RP_BATCH) {
      [[maybe_unused]] const char* const batch_in = in;
      [[maybe_unused]] char* const batch_out = out;
      // 4-bit rows of the batch that the 64-bit way has to decide; of the others, elements that it has to, and their row's scales
      [[maybe_unused]] unsigned again = 0, near[RP_BATCH] = {}, held[RP_BATCH] = {};
      uint4 r0[RP_BATCH], r1[RP_BATCH];
#pragma unroll
      for (int u = 0; u < RP_BATCH; ++u) {
        r0[u] = r1[u] = make_uint4(0u, 0u, 0u, 0u);
        if (h + u < hi && live) {
          r0[u] = *reinterpret_cast<const uint4*>(in + 2 * e0);
          r1[u] = *reinterpret_cast<const uint4*>(in + 2 * e1);
        }
        in += from.head_stride;
      }
#pragma unroll
      for (int u = 0; u < RP_BATCH; ++u) {
        if (h + u >= hi) break;
        if (!quantised && !(turned && kind < 2)) {             // copied bit for bit
          if (live) {
            *reinterpret_cast<uint4*>(out + row_off + 2 * c0) = r0[u];
            *reinterpret_cast<uint4*>(out + row_off + 2 * c1) = r1[u];
          }
          out += out_stride;
          continue;
        }
        float x[16];
        const uint32_t w[8] = {r0[u].x, r0[u].y, r0[u].z, r0[u].w, r1[u].x, r1[u].y, r1[u].z, r1[u].w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 f = dd_unpack2<T>(w[i]);
          x[2 * i] = f.x;
          x[2 * i + 1] = f.y;
        }
        if (kind < 2 && turned) {
          if (a.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float p = x[2 * i], q = x[2 * i + 1];
              x[2 * i] = fmaf(p, cs[i], -q * sn[i]);
              x[2 * i + 1] = fmaf(q, cs[i], p * sn[i]);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float p = x[i], q = x[8 + i];
              x[i] = fmaf(p, cs[i], -q * sn[i]);
              x[8 + i] = fmaf(q, cs[i], p * sn[i]);
            }
          }
        }
        if constexpr (paged && FMT == DD_CACHE_INT4) {
          const rp_place& at = kind == 2 ? plain_place : place;
          // the larger magnitudes compare as unsigned numbers, NaN and infinities above all others
          unsigned top[2] = {0u, 0u};
#pragma unroll
          for (int i = 0; i < 16; ++i) top[i >> 3] = max(top[i >> 3], __float_as_uint(x[i]) & 0x7fffffffu);
          unsigned amax = max(top[0], top[1]);
#pragma unroll
          for (int m = 1; m < LANES; m <<= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, m));
          unsigned group[2];
          if (kind == 2) {
            group[0] = group[1] = max(top[0], top[1]);
          } else if (next_lane) {
            const unsigned n0 = __shfl_xor_sync(0xffffffffu, top[0], 1), n1 = __shfl_xor_sync(0xffffffffu, top[1], 1);
            group[0] = max(top[0], same_lane ? top[1] : n0);
            group[1] = max(top[1], same_lane ? top[0] : n1);
          } else {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const unsigned a0 = __shfl_sync(0xffffffffu, top[0], c ? at.mate1 : at.mate0), a1 = __shfl_sync(0xffffffffu, top[1], c ? at.mate1 : at.mate0);
              group[c] = max(top[c], (at.slots >> c) & 1 ? a1 : a0);
            }
          }
          const bool known = kind == 2 || a.rot16 == 0;        // the row is what was given
          int byte = dd_int4_exponent_byte(__uint_as_float(amax));
          const float up = dd_two_to_byte(254 - byte), whole = __uint_as_float(amax) * up, eps = whole * RP_KNOWN;
          bool slow = amax >= RP_NEAR_MOST || (byte < 8 && amax != 0u);      // (a scale of 2^-4 * 2^(byte - 127) has an inverse from 8 on)
          if (!known) slow |= fabsf(a.amplitude) < RP_LEAST || fabsf(whole - 3136.f) < eps || fabsf(whole - 1568.f) < eps;
          unsigned scale[2];
          uint32_t code[2];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            if (kind == 2 && c == 1) scale[1] = scale[0];
            const float r = rp_seventh(__uint_as_float(group[c]) * up);
            if (!known) slow |= r > 0x1p-4f && rp_near_scale(r, eps * 0.15f);
            const float step = rp_round_e4m3(fmaxf(r, 0x1p-4f), scale[c]);
            const float inv = rp_rcp(step) * up, s1 = step * dd_two_to_byte(byte);
            constexpr float magic = 12582912.f + 8.f;
            uint32_t word = 0;
            if (known) {
#pragma unroll
              for (int i = 7; i >= 0; --i) {
                float q = x[8 * c + i] * inv;
                q = fmaf(fmaf(-q, s1, x[8 * c + i]), inv, q);
                word = (word << 4) + __float_as_uint(q + magic);
              }
            } else {
              const float far = 0.5f - eps * rp_rcp(step);
#pragma unroll
              for (int i = 7; i >= 0; --i) {
                const float t = fmaf(x[8 * c + i], inv, magic);
                if (fabsf(fmaf(x[8 * c + i], inv, magic - t)) > far) near[u] |= 1u << (8 * c + i);
                word = (word << 4) + __float_as_uint(t);
              }
            }
            // the constant part 0x4b400000 of every element, shifted by 4 i
            code[c] = amax == 0u ? 0x88888888u : word - 0x40000000u - 0xb4000000u - 0x4b400000u;
          }
          if (slow && live) again |= 1u << u;
          if (kind < 2) held[u] = (unsigned)byte | scale[0] << 8 | scale[1] << 16;
          if (live) put4(out, scale, code, byte);
          out += out_stride;
          continue;
        }
        if (paged && FMT == DD_CACHE_E4M3) {
          float amax = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) amax = fmaxf(amax, fabsf(x[i]));
#pragma unroll
          for (int m = 1; m < LANES; m <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, m));
          if (amax > 3.4028234e38f) {                          // an infinity (fmaxf passes over NaN): finite values only
            amax = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float v = fabsf(x[i]);
              if (v <= 3.4028234e38f) amax = fmaxf(amax, v);
              else x[i] = __uint_as_float(0x7fc00000u);
            }
#pragma unroll
            for (int m = 1; m < LANES; m <<= 1) amax = fmaxf(amax, __shfl_xor_sync(peers, amax, m));
          }
          const int byte = dd_e4m3_exponent_byte(amax);
          const float inv = dd_two_to_byte(254 - byte);        // 2^(127 - byte): exact, so the code is rounded once
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] *= inv;
          if (live) {
            char* row = out + row_off;
            const uint2 lo8 = make_uint2(dd_float_to_e4m3x4(x[0], x[1], x[2], x[3]), dd_float_to_e4m3x4(x[4], x[5], x[6], x[7]));
            const uint2 hi8 = make_uint2(dd_float_to_e4m3x4(x[8], x[9], x[10], x[11]), dd_float_to_e4m3x4(x[12], x[13], x[14], x[15]));
            if (c1 == c0 + 8) {
              *reinterpret_cast<uint4*>(row + c0) = make_uint4(lo8.x, lo8.y, hi8.x, hi8.y);
            } else {
              *reinterpret_cast<uint2*>(row + c0) = lo8;
              *reinterpret_cast<uint2*>(row + c1) = hi8;
            }
            if (j == 0) out[2 * page_tokens * D + (kind == 2 ? page_tokens : 0) + off] = (char)byte;
          }
        } else if (live) {
          *reinterpret_cast<uint4*>(out + row_off + 2 * c0) =
              make_uint4(dd_pack2<T>(x[0], x[1]), dd_pack2<T>(x[2], x[3]), dd_pack2<T>(x[4], x[5]), dd_pack2<T>(x[6], x[7]));
          *reinterpret_cast<uint4*>(out + row_off + 2 * c1) =
              make_uint4(dd_pack2<T>(x[8], x[9]), dd_pack2<T>(x[10], x[11]), dd_pack2<T>(x[12], x[13]), dd_pack2<T>(x[14], x[15]));
        }
        out += out_stride;
      }
      if constexpr (paged && FMT == DD_CACHE_INT4) {
        again = __reduce_or_sync(peers, again);
        if (kind < 2 && live && a.rot16) {
#pragma unroll 1
          for (int u = 0; u < RP_BATCH; ++u) {
            unsigned m = near[0], k = held[0];
#pragma unroll
            for (int v = 1; v < RP_BATCH; ++v) {
              if (u == v) {
                m = near[v];
                k = held[v];
              }
            }
            if ((again >> u) & 1) m = 0;
            while (m) {
              const int e = __ffs(m) - 1;
              m &= m - 1;
              const uint32_t n = rp_int4_element<T>(batch_in + u * from.head_stride, c0, c1, e, turned ? a.turns : nullptr, pos, a.amplitude, j, a.interleaved, (int)(k & 0xff),
                                                    (k >> (e < 8 ? 8 : 16)) & 0xff);
              uint32_t* word = reinterpret_cast<uint32_t*>(batch_out + u * out_stride + (off >> 4) * dd_int4_tile_bytes(D) + dd_int4_k_at<D>(off & 15, (e < 8 ? c0 : c1) >> 3));
              *word = (*word & ~(15u << (4 * (e & 7)))) | n << (4 * (e & 7));
            }
          }
        }
        while (again) {
          const int u = __ffs(again) - 1;
          again &= again - 1;
          unsigned scale[2];
          uint32_t code[2];
          const int byte = rp_int4_slow<T, D>(batch_in + u * from.head_stride, kind == 2 ? plain_place : place, turned && kind < 2 ? a.turns : nullptr, pos,
                                              a.amplitude, j, a.interleaved, peers, scale, code);
          if (live) put4(batch_out + u * out_stride, scale, code, byte);
        }
      }
    }
  };
  rows(std::integral_constant<int, 0>(), h0, min(h1, a.n_q), a.q, a.q_out);
  rows(std::integral_constant<int, 1>(), max(h0 - a.n_q, 0), min(h1 - a.n_q, a.n_k), a.k, a.k_out);
  if (FMT >= 0) rows(std::integral_constant<int, 2>(), max(h0 - a.n_q - a.n_k, 0), h1 - a.n_q - a.n_k, a.v, a.v);
}

template <typename T, int D>
const void* rp_kernel_of(int fmt) {
  if (fmt < 0) return (const void*)dd_rope_kernel<T, D, -1>;
  if (fmt == DD_CACHE_E4M3) return (const void*)dd_rope_kernel<T, D, DD_CACHE_E4M3>;
  if (fmt == DD_CACHE_INT4) return (const void*)dd_rope_kernel<T, D, DD_CACHE_INT4>;
  return (const void*)dd_rope_kernel<T, D, DD_CACHE_BF16>;      // 16-bit pages of the rows' own type
}

int rp_launch(rp_args& a, int head_dim, int dtype, int fmt, cudaStream_t st, const char* who, int device) {
  const int lanes = head_dim / 16, per_warp = 32 / lanes;
  const int n_heads = a.n_q + a.n_k * (fmt >= 0 ? 2 : 1);
  // Heads per group of lanes: 8 (two batches of loads, the token's angles computed once per 8 rows) while that gives half the
  // groups that fill the device, fewer for fewer tokens. 32768 tokens of 40 heads: 8 heads 102.6 us, 16 heads 105.9, 4 heads 114.7; into
  // 16-bit pages, unturned, 8 heads 47.5, 16 heads 51.2. Rows that are quantised on the way 16: e4m3 8 heads 123.8, 16 heads 120.0, 24
  // 122.8; 4-bit 176.7, 163.3, 163.6.
  int sms = 0;
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
  if (sms <= 0) sms = 148;
  const long long fill = (long long)sms * rp_blocks(fmt) * RP_THREADS / lanes;
  a.slice_heads = (fmt == DD_CACHE_E4M3 || fmt == DD_CACHE_INT4 ? 4 : 2) * RP_BATCH;
  while (a.slice_heads > 1 && (long long)a.n_tokens * ((n_heads + a.slice_heads - 1) / a.slice_heads) < fill / 2) a.slice_heads /= 2;
  a.slices = (n_heads + a.slice_heads - 1) / a.slice_heads;
  const long long per_block = (long long)(RP_THREADS / 32) * per_warp;
  const long long blocks = ((long long)a.n_tokens + per_block - 1) / per_block * a.slices;
  if (blocks > 0x7fffffffLL) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: too many tokens", who);
  const void* f = head_dim == 128 ? (dtype == DD_BF16 ? rp_kernel_of<__nv_bfloat16, 128>(fmt) : rp_kernel_of<__half, 128>(fmt))
                                  : (dtype == DD_BF16 ? rp_kernel_of<__nv_bfloat16, 64>(fmt) : rp_kernel_of<__half, 64>(fmt));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(RP_THREADS);
  cfg.stream = st;
  cudaLaunchAttribute at;
  dd_pdl_attr(&at);
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  void* args[] = {&a};
  return dd_launch(who, &cfg, f, args);
}

rp_rows rp_of(const dd_rows* r) {
  rp_rows o = {nullptr, 0, 0};
  if (r) { o.data = (char*)r->data; o.token_stride = r->token_stride * 2; o.head_stride = r->head_stride * 2; }
  return o;
}

}  // namespace

extern "C" int dd_rope_turns(int rot_dim, double base, int scaling, double factor, double original_len, double low_turns,
                             double high_turns, double* turns) {
  const char* who = "dd_rope_turns";
  if (!turns) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: turns is NULL", who);
  if (rot_dim < 16 || rot_dim > 128 || rot_dim % 16) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: rot_dim must be a multiple of 16 in [16, 128]", who);
  if (!(base > 1.0) || !isfinite(base)) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: base must be above 1", who);
  if (scaling < DD_ROPE_NONE || scaling > DD_ROPE_BY_PARTS) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: unknown scaling", who);
  if (scaling != DD_ROPE_NONE && (!(factor > 0.0) || !isfinite(factor))) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: factor must be positive", who);
  if (scaling == DD_ROPE_BY_PARTS && (!(original_len > 0.0) || !isfinite(original_len) || !(high_turns > low_turns) || !isfinite(high_turns) || !isfinite(low_turns)))
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: need original_len > 0 and high_turns > low_turns", who);
  const double two_pi = 6.283185307179586476925286766559;
  if (scaling == DD_ROPE_NTK) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
  for (int i = 0; i < rot_dim / 2; ++i) {
    double t = pow(base, -2.0 * i / rot_dim) / two_pi;
    if (scaling == DD_ROPE_LINEAR) t /= factor;
    if (scaling == DD_ROPE_BY_PARTS) {
      double kept = (original_len * t - low_turns) / (high_turns - low_turns);
      kept = kept < 0.0 ? 0.0 : (kept > 1.0 ? 1.0 : kept);
      t = (1.0 - kept) * t / factor + kept * t;
    }
    turns[i] = t;
  }
  return DD_OK;
}

int dd_check_rope(const dd_rope* r, const char* who, int head_dim) {
  if (r->rot_dim < 16 || r->rot_dim > head_dim || r->rot_dim % 16)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: rot_dim must be a multiple of 16 in [16, head_dim]", who);
  if (r->layout != DD_ROPE_HALF && r->layout != DD_ROPE_INTERLEAVED) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: unknown rotary layout", who);
  if (!isfinite(r->amplitude)) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: amplitude is not finite", who);
  if (!r->turns) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: rope->turns is NULL", who);
  return DD_OK;
}

static int rp_check_pair(const dd_rows* in, const dd_rows* out, const char* who, const char* name, const char* name_out, int head_dim, int n_tokens) {
  if (!in != !out) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: %s and %s go together", who, name, name_out);
  if (!in) return DD_OK;
  DD_TRY(dd_check_rows(in, who, name, head_dim, n_tokens, false));
  DD_TRY(dd_check_rows(out, who, name_out, head_dim, n_tokens, true));
  if (in->n_heads != out->n_heads || in->dtype != out->dtype)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: %s and %s differ in heads or type", who, name, name_out);
  return DD_OK;
}

extern "C" int dd_rope_apply(const dd_rope* rope, int head_dim, int n_tokens, const int* positions, const dd_rows* q,
                             const dd_rows* k, const dd_rows* q_out, const dd_rows* k_out, int backward, void* stream) {
  const char* who = "dd_rope_apply";
  if (!rope) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: rope is NULL", who);
  if (head_dim != 64 && head_dim != 128) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: head_dim must be 64 or 128", who);
  if (n_tokens < 0) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: n_tokens is negative", who);
  if (backward != 0 && backward != 1) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: backward must be 0 or 1", who);
  if (!q && !k) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: neither q nor k is given", who);
  DD_TRY(dd_check_rope(rope, who, head_dim));
  if (n_tokens == 0) return DD_OK;
  DD_TRY(rp_check_pair(q, q_out, who, "q", "q_out", head_dim, n_tokens));
  DD_TRY(rp_check_pair(k, k_out, who, "k", "k_out", head_dim, n_tokens));
  if (q && k && q->dtype != k->dtype) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: q and k differ in type", who);
  const int device = dd_current_device();
  DD_TRY(dd_check_ptr(rope->turns, who, "rope->turns", 8, device));
  DD_TRY(dd_check_ptr(positions, who, "positions", 4, device));
  if (q) DD_TRY(dd_check_ptr(q->data, who, "q", 16, device));
  if (q) DD_TRY(dd_check_ptr(q_out->data, who, "q_out", 16, device));
  if (k) DD_TRY(dd_check_ptr(k->data, who, "k", 16, device));
  if (k) DD_TRY(dd_check_ptr(k_out->data, who, "k_out", 16, device));
  rp_args a = {};
  a.turns = rope->turns;
  a.positions = positions;
  a.q = rp_of(q); a.k = rp_of(k); a.q_out = rp_of(q_out); a.k_out = rp_of(k_out);
  a.n_tokens = n_tokens;
  a.n_q = q ? q->n_heads : 0;
  a.n_k = k ? k->n_heads : 0;
  a.rot16 = rope->rot_dim / 16;
  a.interleaved = rope->layout == DD_ROPE_INTERLEAVED;
  a.backward = backward;
  a.amplitude = rope->amplitude;
  return rp_launch(a, head_dim, q ? q->dtype : k->dtype, -1, (cudaStream_t)stream, who, device);
}

extern "C" int dd_cache_append(const dd_cache* cache, int n_tokens, const int* positions, const int* requests,
                               const dd_rows* k, const dd_rows* v, const dd_rope* rope, const dd_rows* q,
                               const dd_rows* q_out, void* stream) {
  const char* who = "dd_cache_append";
  DD_TRY(dd_check_cache(cache, who));
  if (n_tokens < 0) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: n_tokens is negative", who);
  if (!requests && n_tokens % cache->batch)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: without requests, n_tokens (%d) must be a multiple of batch (%d)", who, n_tokens, cache->batch);
  if ((q || q_out) && !rope) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: q is turned with rope, which is NULL", who);
  if (rope) DD_TRY(dd_check_rope(rope, who, cache->head_dim));
  if (n_tokens == 0) return DD_OK;
  DD_TRY(dd_check_rows(k, who, "k", cache->head_dim, n_tokens, false));
  DD_TRY(dd_check_rows(v, who, "v", cache->head_dim, n_tokens, false));
  if (k->n_heads != cache->n_kv_heads || v->n_heads != cache->n_kv_heads)
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: k and v must have the cache's %d heads", who, cache->n_kv_heads);
  if (k->dtype != v->dtype) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: k and v differ in type", who);
  if ((cache->format == DD_CACHE_BF16 && k->dtype != DD_BF16) || (cache->format == DD_CACHE_FP16 && k->dtype != DD_FP16))
    return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: a 16-bit cache takes rows of its own type", who);
  DD_TRY(rp_check_pair(q, q_out, who, "q", "q_out", cache->head_dim, n_tokens));
  if (q && q->dtype != k->dtype) return dd_fail(nullptr, DD_ERR_INVALID_ARG, "%s: q and k differ in type", who);
  const int device = dd_current_device();
  const char* data = nullptr;
  DD_TRY(dd_check_cache_memory(cache, who, device, true, &data, nullptr));
  DD_TRY(dd_check_ptr(positions, who, "positions", 4, device));
  if (requests) DD_TRY(dd_check_ptr(requests, who, "requests", 4, device));
  DD_TRY(dd_check_ptr(k->data, who, "k", 16, device));
  DD_TRY(dd_check_ptr(v->data, who, "v", 16, device));
  if (rope) DD_TRY(dd_check_ptr(rope->turns, who, "rope->turns", 8, device));
  if (q) DD_TRY(dd_check_ptr(q->data, who, "q", 16, device));
  if (q) DD_TRY(dd_check_ptr(q_out->data, who, "q_out", 16, device));
  rp_args a = {};
  a.turns = rope ? rope->turns : nullptr;
  a.positions = positions;
  a.requests = requests;
  a.q = rp_of(q); a.k = rp_of(k); a.v = rp_of(v); a.q_out = rp_of(q_out);
  a.n_tokens = n_tokens;
  a.n_q = q ? q->n_heads : 0;
  a.n_k = cache->n_kv_heads;
  a.rot16 = rope ? rope->rot_dim / 16 : 0;
  a.interleaved = rope && rope->layout == DD_ROPE_INTERLEAVED;
  a.amplitude = rope ? rope->amplitude : 1.f;
  a.tokens_per_request = requests ? 1 : n_tokens / cache->batch;
  a.cache = dd_make_view(cache, data);
  return rp_launch(a, cache->head_dim, k->dtype, cache->format == DD_CACHE_E4M3 || cache->format == DD_CACHE_INT4 ? cache->format : DD_CACHE_BF16,
                   (cudaStream_t)stream, who, device);
}
