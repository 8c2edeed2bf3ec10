/* Decode attention over the pages that a cheap score selects: bounds of a page's
 * keys, the bound of its logits, the selection, and the attention over it. */
#include <cuda_bf16.h>

#include <math.h>
#include <string.h>

#include "md_internal.h"
#include "md_ptx.cuh"

namespace md {

namespace {

constexpr uint32_t POS_INF2 = 0x7F807F80u, NEG_INF2 = 0xFF80FF80u;   // two bf16

__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {   // NaN if either is
  uint32_t r;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

/* Physical id of sequence b's page pg, or -1: not a page of the sequence, or a
 * table entry outside the pool. */
__device__ __forceinline__ int page_id(const PageSet &p, int b, int pg) {
  if ((unsigned)pg >= (unsigned)p.n_pages[b]) return -1;
  const int phys = p.block_table[(size_t)b * p.P_max + pg];
  return (unsigned)phys < (unsigned)p.P_phys ? phys : -1;
}
/* Its tokens. */
__device__ __forceinline__ int page_tokens(const PageSet &p, int b, int pg) {
  const int n = p.page_fill ? p.page_fill[(size_t)b * p.P_max + pg] : p.n_tokens[b] - pg * p.ps;
  return n < p.ps ? n : p.ps;
}

/* ------------------------------------------------------------- bounds --- */
/* A warp per (layer, page, KV head): half a warp per K row, 16 bytes per lane. */
template <int PS>
__global__ void __launch_bounds__(256) bounds_kernel(const __grid_constant__ BoundsParams p) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, j = lane & 15, odd = lane >> 4;
  const long long total = p.start[p.n_seqs], units = total * p.L * p.Hkv;
  for (long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += (long long)gridDim.x * 8) {
    const int h = (int)(u % p.Hkv);
    const long long r = u / p.Hkv;
    const int l = (int)(r / total), at = (int)(r - l * total);
    int b = 0, hi = p.n_seqs;          // the sequence: start[b] <= at < start[b + 1]
    while (hi - b > 1) {
      const int mid = (b + hi) >> 1;
      if (p.start[mid] <= at) b = mid;
      else hi = mid;
    }
    const int pg = p.first[b] + at - p.start[b];
    const int phys = page_id(p, b, pg);
    if (phys < 0) continue;            // the whole warp
    const int n = page_tokens(p, b, pg);
    const size_t page = ((size_t)l * p.P_phys + phys) * p.Hkv + h;
    const uint4 *src = (const uint4 *)(p.pool + page * 2 * PS * D) + j;
    uint32_t lo[4], hi4[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = POS_INF2;
      hi4[i] = NEG_INF2;
    }
#pragma unroll
    for (int i = 0; i < PS / 2; ++i) {
      const int row = 2 * i + odd;
      if (row < n) {
        const uint4 x = src[row * 16];
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          lo[k] = min2(lo[k], w[k]);
          hi4[k] = max2(hi4[k], w[k]);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      lo[k] = min2(lo[k], __shfl_xor_sync(0xffffffffu, lo[k], 16));
      hi4[k] = max2(hi4[k], __shfl_xor_sync(0xffffffffu, hi4[k], 16));
    }
    uint4 *dst = (uint4 *)(p.bounds + page * 2 * D) + lane;
    *dst = odd ? make_uint4(hi4[0], hi4[1], hi4[2], hi4[3]) : make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
}

/* ------------------------------------------------------------- scores --- */
/* In the MMAs of this file the summed dimension is permuted alike in both
 * operands: lane (g, t) takes 8 consecutive channels 32 j + 8 t .. of its rows
 * with one 16-byte load, and the four words are the fragments of two MMAs. */

/* The B fragments of 8 query heads (columns): words j * 4 .. j * 4 + 3 are the
 * channels 32 j + 8 t .. of head g; padded heads are zero. */
__device__ __forceinline__ void load_q(const uint16_t *q, int G, int g, int t, uint32_t (&w)[16]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint4 x = g < G ? *((const uint4 *)(q + (size_t)g * D) + 4 * j + t) : make_uint4(0, 0, 0, 0);
    w[4 * j] = x.x;
    w[4 * j + 1] = x.y;
    w[4 * j + 2] = x.z;
    w[4 * j + 3] = x.w;
  }
}

/* A warp per 16 pages of a (sequence, layer, KV head): the pages are an MMA's
 * rows, the query heads its columns, and lo and hi side by side the summed
 * dimension, against the queries' negative and positive parts. */
__global__ void __launch_bounds__(256) page_scores_kernel(const __grid_constant__ PageScoresParams p, int most) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int lh = p.L * p.Hkv;
  const long long units = (long long)p.n_seqs * lh * most;   // most: 16-page tiles of the longest sequence
  const long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (u >= units) return;
  const long long row = u / most;
  const int tile = (int)(u - row * most);
  const int b = (int)(row / lh), l = (int)(row % lh) / p.Hkv, h = (int)(row % p.Hkv);
  const int P = p.n_pages[b];
  if (tile * 16 >= P) return;
  uint32_t q[16];
  load_q(p.q + (((size_t)b * p.L + l) * p.Hq + h * p.G) * D, p.G, g, t, q);
  const int p0 = tile * 16 + g, p1 = p0 + 8;
  const int i0 = page_id(p, b, p0), i1 = page_id(p, b, p1);
  const uint4 *s0 = (const uint4 *)(p.bounds + (((size_t)l * p.P_phys + (i0 < 0 ? 0 : i0)) * p.Hkv + h) * 2 * D) + t;
  const uint4 *s1 = (const uint4 *)(p.bounds + (((size_t)l * p.P_phys + (i1 < 0 ? 0 : i1)) * p.Hkv + h) * 2 * D) + t;
  float c[4] = {0.f, 0.f, 0.f, 0.f};
  const uint4 none = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int j = 0; j < 8; ++j) {   // 0..3: lo, 4..7: hi
    const uint4 x = i0 >= 0 ? s0[4 * j] : none, y = i1 >= 0 ? s1[4 * j] : none;
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = j < 4 ? min2(q[4 * (j & 3) + k], 0u) : max2(q[4 * (j & 3) + k], 0u);
    mma_bf16(c, x.x, y.x, x.y, y.y, w[0], w[1]);
    mma_bf16(c, x.z, y.z, x.w, y.w, w[2], w[3]);
  }
  /* columns 2t, 2t + 1 of rows g (c[0], c[1]) and g + 8 */
  const bool in0 = 2 * t < p.G, in1 = 2 * t + 1 < p.G;
  auto top = [](float x, float y) { return x != x || y != y ? NAN : fmaxf(x, y); };
  float m0 = in0 ? (in1 ? top(c[0], c[1]) : c[0]) : -INFINITY, m1 = in0 ? (in1 ? top(c[2], c[3]) : c[2]) : -INFINITY;
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    m0 = top(m0, __shfl_xor_sync(0xffffffffu, m0, o));
    m1 = top(m1, __shfl_xor_sync(0xffffffffu, m1, o));
  }
  float *dst = p.scores + (size_t)row * p.P_max;
  if (t == 0 && p0 < P) dst[p0] = m0 * p.scale;
  if (t == 0 && p1 < P) dst[p1] = m1 * p.scale;
}

/* ---------------------------------------------------------------- top --- */
/* fp32 -> uint32 in the same order; NaN above all, the zeros equal */
__device__ __forceinline__ uint32_t score_key(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

/* A block per row: radix select of the k-th largest key, eight bits at a time,
 * then an ordered write of the pages above it and of the first ones equal to it. */
constexpr int TOP_THREADS = 512;
__global__ void __launch_bounds__(TOP_THREADS) page_top_kernel(const __grid_constant__ PageTopParams p) {
  __shared__ int hist[256], warp_gt[TOP_THREADS / 32], warp_eq[TOP_THREADS / 32];
  __shared__ uint32_t s_prefix;
  __shared__ int s_k;
  pdl_wait();
  pdl_trigger();
  const long long row = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int P = p.n_pages[row / p.rows];
  const float *sc = p.scores + row * p.P_max;
  int32_t *out = p.ids + row * p.top;
  if (P <= p.top) {
    for (int i = tid; i < p.top; i += TOP_THREADS) out[i] = i < P ? i : -1;
    return;
  }
  const int lo = p.first, hi = P - p.last;     // the pages to choose from
  const int k = p.top - p.first - p.last;
  for (int i = tid; i < p.first; i += TOP_THREADS) out[i] = i;
  for (int i = tid; i < p.last; i += TOP_THREADS) out[p.top - p.last + i] = hi + i;
  if (k == 0) return;
  uint32_t prefix = 0, mask = 0;
  int left = k;                                // still to be taken among the keys that match the prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += TOP_THREADS) hist[i] = 0;
    __syncthreads();
    for (int i = lo + tid; i < hi; i += TOP_THREADS) {
      const uint32_t key = score_key(sc[i]);
      if ((key & mask) == prefix) atomicAdd(&hist[key >> shift & 255], 1);
    }
    __syncthreads();
    if (tid < 32) {                            // the digit of the left-th largest: bins from the top, eight per lane
      int c[8], sum = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += c[i] = hist[255 - 8 * lane - i];
      int incl = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      int before = incl - sum;
      if (before < left && left <= incl) {
        int i = 0;
        while (before + c[i] < left) before += c[i++];
        s_prefix = prefix | (uint32_t)(255 - 8 * lane - i) << shift;
        s_k = left - before;
      }
    }
    __syncthreads();
    prefix = s_prefix;
    left = s_k;
    mask |= 255u << shift;
    __syncthreads();
  }
  int done_gt = 0, done_eq = 0;
  for (int base = lo; base < hi; base += TOP_THREADS) {
    const int i = base + tid;
    const uint32_t key = i < hi ? score_key(sc[i]) : 0;
    const bool gt = i < hi && key > prefix, eq = i < hi && key == prefix;
    const unsigned mg = __ballot_sync(0xffffffffu, gt), me = __ballot_sync(0xffffffffu, eq);
    if (lane == 0) {
      warp_gt[warp] = __popc(mg);
      warp_eq[warp] = __popc(me);
    }
    __syncthreads();
    int g = done_gt + __popc(mg & ((1u << lane) - 1)), e = done_eq + __popc(me & ((1u << lane) - 1));
    int tg = 0, te = 0;
    for (int w = 0; w < TOP_THREADS / 32; ++w) {
      if (w < warp) {
        g += warp_gt[w];
        e += warp_eq[w];
      }
      tg += warp_gt[w];
      te += warp_eq[w];
    }
    if (gt || (eq && e < left)) out[p.first + g + min(e, left)] = i;
    done_gt += tg;
    done_eq += te;
    __syncthreads();
  }
}

/* ------------------------------------------------------------- attend --- */
/* A block per (sequence, layer, KV head).  A warp takes 16 tokens of a page at
 * a time, straight from global memory into MMA fragments:
 *   S = K Q^T   rows are tokens, columns the group's heads
 *   O^T = V^T P^T  rows are channels, summed over the tokens
 * A lane's V words hold two neighbouring channels of one token; exchanging
 * halves with the next token's word makes the fragments of two rows. */
constexpr int AT_WARPS = 8;

struct Tile {
  uint4 k[8];   // rows g and g + 8: 16 bytes at channels 32 j + 8 t
  uint4 v[8];   // tokens 2t, 2t + 1, 2t + 8, 2t + 9: channels 8 g .. and 64 + 8 g ..
};

__device__ __forceinline__ void load_k(const uint16_t *page, int valid, int g, int t, uint4 (&k)[8]) {
  const uint4 none = make_uint4(0, 0, 0, 0);
  const uint4 *r = (const uint4 *)(page + (size_t)g * D) + t;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    k[2 * j] = g < valid ? r[4 * j] : none;
    k[2 * j + 1] = g + 8 < valid ? r[4 * j + 16 * 8] : none;
  }
}
__device__ __forceinline__ void load_v(const uint16_t *page, int valid, int g, int t, uint4 (&v)[8]) {
  const uint4 none = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int tok = 2 * t + (i & 1) + 8 * (i >> 1);
    const uint4 *r = (const uint4 *)(page + (size_t)tok * D) + g;
    v[2 * i] = tok < valid ? r[0] : none;
    v[2 * i + 1] = tok < valid ? r[8] : none;
  }
}
/* c[0], c[1]: token g, heads 2t, 2t + 1; c[2], c[3]: token g + 8 */
__device__ __forceinline__ void tile_scores(const uint4 (&k)[8], const uint32_t (&q)[16], float scale, int valid, int g,
                                            float (&c)[4]) {
  float c2[4] = {0.f, 0.f, 0.f, 0.f};
  c[0] = c[1] = c[2] = c[3] = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint4 &x = k[2 * j], &y = k[2 * j + 1];
    mma_bf16(c, x.x, y.x, x.y, y.y, q[4 * j], q[4 * j + 1]);
    mma_bf16(c2, x.z, y.z, x.w, y.w, q[4 * j + 2], q[4 * j + 3]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = g + 8 * (i >> 1) < valid ? (c[i] + c2[i]) * scale : -INFINITY;
}

__global__ void __launch_bounds__(32 * AT_WARPS) attend_pages_kernel(const __grid_constant__ AttendPagesParams p) {
  __shared__ float sm[AT_WARPS][GP], sl[AT_WARPS][GP], so[AT_WARPS][GP][D + 4];
  __shared__ float fm[GP], fz[GP];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const long long row = blockIdx.x;
  const int lh = p.L * p.Hkv;
  const int b = (int)(row / lh), l = (int)(row % lh) / p.Hkv, h = (int)(row % p.Hkv);
  const int tpp = p.ps / TILE, tiles = p.top * tpp;
  const int32_t *ids = p.ids + row * p.top;
  const size_t q_row = ((size_t)b * p.L + l) * p.Hq + h * p.G;
  uint32_t q[16];
  load_q(p.q + q_row * D, p.G, g, t, q);
  /* a tile's K rows, or null, and its tokens */
  auto tile_at = [&](int tile, int &valid) -> const uint16_t * {
    const int pg = ids[tile / tpp], phys = page_id(p, b, pg), sub = tile % tpp * TILE;
    valid = 0;
    if (phys < 0) return nullptr;
    valid = min(TILE, page_tokens(p, b, pg) - sub);
    return p.pool + ((((size_t)l * p.P_phys + phys) * p.Hkv + h) * 2 * p.ps + sub) * D;
  };
  float m[2] = {-INFINITY, -INFINITY}, z[2] = {0.f, 0.f}, o[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  for (int tile = warp; tile < tiles; tile += AT_WARPS) {
    int valid;
    const uint16_t *page = tile_at(tile, valid);
    if (valid <= 0) continue;
    Tile x;
    load_k(page, valid, g, t, x.k);
    load_v(page + (size_t)p.ps * D, valid, g, t, x.v);
    float c[4];
    tile_scores(x.k, q, p.scale_log2, valid, g, c);
    float mx[2] = {fmaxf(c[0], c[2]), fmaxf(c[1], c[3])};
#pragma unroll
    for (int s = 4; s < 32; s <<= 1)
#pragma unroll
      for (int i = 0; i < 2; ++i) mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], s));
    float base[2], alpha[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float n = fmaxf(m[i], mx[i]);
      base[i] = n == -INFINITY ? 0.f : n;     // nothing but -inf so far: weights 0
      alpha[i] = exp2f(m[i] - base[i]);
      m[i] = n;
    }
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = exp2f(c[i] - base[i & 1]);
    z[0] = z[0] * alpha[0] + w[0] + w[2];
    z[1] = z[1] * alpha[1] + w[1] + w[3];
    uint32_t hi[2], lo[2];                    // each weight as two bf16: 16 bits of it enter the product
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t u = pack_bf16(w[2 * i], w[2 * i + 1]);
      hi[i] = movmatrix_trans(u);
      lo[i] = movmatrix_trans(pack_bf16(w[2 * i] - __uint_as_float(u << 16), w[2 * i + 1] - __uint_as_float(u & 0xffff0000u)));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint4 *v = x.v + (i >> 2);
      auto word = [&](int tok) { return ((const uint32_t *)&v[2 * tok])[i & 3]; };
      const uint32_t a0 = __byte_perm(word(0), word(1), 0x5410), a1 = __byte_perm(word(0), word(1), 0x7632),
                     a2 = __byte_perm(word(2), word(3), 0x5410), a3 = __byte_perm(word(2), word(3), 0x7632);
      o[i][0] *= alpha[0];
      o[i][1] *= alpha[1];
      o[i][2] *= alpha[0];
      o[i][3] *= alpha[1];
      mma_bf16(o[i], a0, a1, a2, a3, hi[0], hi[1]);
      mma_bf16(o[i], a0, a1, a2, a3, lo[0], lo[1]);
    }
  }
#pragma unroll
  for (int s = 4; s < 32; s <<= 1)
#pragma unroll
    for (int i = 0; i < 2; ++i) z[i] += __shfl_xor_sync(0xffffffffu, z[i], s);
  if (g == 0)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sm[warp][2 * t + i] = m[i];
      sl[warp][2 * t + i] = z[i];
    }
#pragma unroll
  for (int i = 0; i < 8; ++i) {               // channels of o[i]: rows g and g + 8
    const int d = (i >> 2) * 64 + 8 * g + 2 * (i & 3);
#pragma unroll
    for (int k = 0; k < 2; ++k) *(float2 *)&so[warp][2 * t + k][d] = make_float2(o[i][k], o[i][2 + k]);
  }
  __syncthreads();
  const int head = threadIdx.x >> 5;          // 8 warps: a head each, 4 channels per lane
  {
    float top = -INFINITY, sum = 0.f;
    for (int w = 0; w < AT_WARPS; ++w) top = fmaxf(top, sm[w][head]);
    const float base = top == -INFINITY ? 0.f : top;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w = 0; w < AT_WARPS; ++w) {
      const float f = exp2f(sm[w][head] - base);
      const float4 y = *(const float4 *)&so[w][head][4 * lane];
      sum += f * sl[w][head];
      acc.x += f * y.x;
      acc.y += f * y.y;
      acc.z += f * y.z;
      acc.w += f * y.w;
    }
    const float r = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);   // no token: zeros; NaN stays
    if (head < p.G)
      *(uint2 *)(p.out + (q_row + head) * D + 4 * lane) =
          make_uint2(pack_bf16(acc.x * r, acc.y * r), pack_bf16(acc.z * r, acc.w * r));
    if (lane == 0) {
      fm[head] = base;
      fz[head] = head < p.G ? r : 0.f;
    }
  }
  if (!p.mass && !p.mass_acc) return;
  __syncthreads();
  float *mass = p.mass + row * p.top * p.ps;
  const uint64_t keep = policy_evict_last();
  const float m0 = fm[2 * t], m1 = fm[2 * t + 1], r0 = fz[2 * t], r1 = fz[2 * t + 1];
  for (int tile = warp; tile < tiles; tile += AT_WARPS) {
    int valid;
    const uint16_t *page = tile_at(tile, valid);
    float w0 = 0.f, w1 = 0.f;
    if (valid > 0) {
      uint4 k[8];
      float c[4];
      load_k(page, valid, g, t, k);
      tile_scores(k, q, p.scale_log2, valid, g, c);
      w0 = (r0 != 0.f ? exp2f(c[0] - m0) * r0 : 0.f) + (r1 != 0.f ? exp2f(c[1] - m1) * r1 : 0.f);
      w1 = (r0 != 0.f ? exp2f(c[2] - m0) * r0 : 0.f) + (r1 != 0.f ? exp2f(c[3] - m1) * r1 : 0.f);
    }
#pragma unroll
    for (int s = 1; s < 4; s <<= 1) {
      w0 += __shfl_xor_sync(0xffffffffu, w0, s);
      w1 += __shfl_xor_sync(0xffffffffu, w1, s);
    }
    if (t == 0 && p.mass) {
      mass[tile * TILE + g] = w0;
      mass[tile * TILE + 8 + g] = w1;
    }
    if (t == 0 && p.mass_acc && valid > 0) {
      unsigned long long *acc = p.mass_acc + (size_t)page_id(p, b, ids[tile / tpp]) * p.ps + tile % tpp * TILE;
      if (g < valid) red_add_u64_hint(acc + g, __float2ull_rn(w0 * MASS_SCALE), keep);
      if (g + 8 < valid) red_add_u64_hint(acc + g + 8, __float2ull_rn(w1 * MASS_SCALE), keep);
    }
  }
}

}  // namespace

cudaError_t launch_bounds(const BoundsParams &p, cudaStream_t s) {
  const long long units = (long long)p.start[p.n_seqs] * p.L * p.Hkv;
  if (units == 0) return cudaSuccess;
  const long long blocks = (units + 7) / 8;
  const int grid = (int)(blocks < (1 << 20) ? blocks : 1 << 20);
  return p.ps == 16 ? launch_pdl(bounds_kernel<16>, grid, 256, 0, s, p) : launch_pdl(bounds_kernel<32>, grid, 256, 0, s, p);
}

cudaError_t launch_page_scores(const PageScoresParams &p, cudaStream_t s) {
  int most = 0;
  for (int b = 0; b < p.n_seqs; ++b) most = p.n_pages[b] > most ? p.n_pages[b] : most;
  most = (most + 15) / 16;
  const long long blocks = ((long long)p.n_seqs * p.L * p.Hkv * most + 7) / 8;
  if (blocks == 0) return cudaSuccess;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(256);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, page_scores_kernel, p, most);
}

cudaError_t launch_page_top(const PageTopParams &p, cudaStream_t s) {
  return launch_pdl(page_top_kernel, p.n_seqs * p.rows, TOP_THREADS, 0, s, p);
}

cudaError_t launch_attend_pages(const AttendPagesParams &p, cudaStream_t s) {
  return launch_pdl(attend_pages_kernel, p.n_seqs * p.L * p.Hkv, 32 * AT_WARPS, 0, s, p);
}

namespace {

/* The checks that the calls share, and what their launches share (Hq: 0 where
 * a call has no queries). */
bool page_set(PageSet &p, const int32_t *block_table, const int32_t *n_tokens, int batch, int L, int Hq, int Hkv, int ps,
              int P_max, int P_phys) {
  if (!n_tokens || batch < 1 || batch > MD_MAX_BATCH || L < 1 || L > 255 || Hkv < 1 || (ps != 16 && ps != 32) ||
      P_max < 1 || P_phys < 1 || (long long)P_max * ps > (long long)MD_MAX_CHUNKS * MD_MAX_CHUNK_TOKENS)
    return false;
  if (Hq && (Hq < Hkv || Hq % Hkv || Hq / Hkv > MD_MAX_GROUP)) return false;
  if ((long long)L * P_phys * Hkv * 2 * ps >= (1LL << 31) || (long long)batch * L * Hkv >= (1LL << 31)) return false;
  p.block_table = block_table;
  p.page_fill = nullptr;
  p.L = L;
  p.Hq = Hq;
  p.Hkv = Hkv;
  p.G = Hq / Hkv;
  p.ps = ps;
  p.P_phys = P_phys;
  p.P_max = P_max;
  p.n_seqs = batch;
  for (int b = 0; b < batch; ++b) {
    if (n_tokens[b] < 0 || n_tokens[b] > P_max * ps) return false;
    p.n_tokens[b] = n_tokens[b];
    p.n_pages[b] = (n_tokens[b] + ps - 1) / ps;
  }
  return true;
}

bool misaligned(const void *p) { return !p || ((uintptr_t)p & 15); }

}  // namespace

}  // namespace md

#define MD_API extern "C" __attribute__((visibility("default")))

MD_API md_status md_page_bounds(const void *pool, const int32_t *block_table, const int32_t *n_tokens,
                                const int32_t *first_page, void *bounds, int batch, int num_layers, int num_kv_heads,
                                int page_size, int max_pages_per_seq, int num_phys_pages, void *stream) {
  using namespace md;
  BoundsParams p;
  if (misaligned(pool) || misaligned(bounds) || !block_table ||
      !page_set(p, block_table, n_tokens, batch, num_layers, 0, num_kv_heads, page_size, max_pages_per_seq,
                num_phys_pages))
    return MD_ERR_INVALID_ARG;
  p.pool = (const uint16_t *)pool;
  p.bounds = (uint16_t *)bounds;
  p.start[0] = 0;
  for (int b = 0; b < batch; ++b) {
    p.first[b] = first_page ? first_page[b] : 0;
    if (p.first[b] < 0) return MD_ERR_INVALID_ARG;
    p.start[b + 1] = p.start[b] + (p.n_pages[b] > p.first[b] ? p.n_pages[b] - p.first[b] : 0);
  }
  return launch_bounds(p, (cudaStream_t)stream) == cudaSuccess ? MD_OK : MD_ERR_CUDA;
}

MD_API md_status md_page_scores(const void *q, const void *bounds, const int32_t *block_table, const int32_t *n_tokens,
                                float *scores, int batch, int num_layers, int num_q_heads, int num_kv_heads,
                                int page_size, int max_pages_per_seq, int num_phys_pages, void *stream) {
  using namespace md;
  PageScoresParams p;
  if (misaligned(q) || misaligned(bounds) || !block_table || !scores || num_q_heads < 1 ||
      !page_set(p, block_table, n_tokens, batch, num_layers, num_q_heads, num_kv_heads, page_size, max_pages_per_seq,
                num_phys_pages))
    return MD_ERR_INVALID_ARG;
  p.q = (const uint16_t *)q;
  p.bounds = (const uint16_t *)bounds;
  p.scores = scores;
  p.scale = (float)(1.0 / sqrt((double)D));
  return launch_page_scores(p, (cudaStream_t)stream) == cudaSuccess ? MD_OK : MD_ERR_CUDA;
}

MD_API md_status md_page_top(const float *scores, const int32_t *n_tokens, int32_t *ids, int batch, int num_layers,
                             int num_kv_heads, int page_size, int max_pages_per_seq, int top_pages, int first_pages,
                             int last_pages, void *stream) {
  using namespace md;
  PageSet s;
  if (!scores || !ids || top_pages < 1 || first_pages < 0 || last_pages < 0 || first_pages > top_pages ||
      last_pages > top_pages - first_pages ||
      !page_set(s, nullptr, n_tokens, batch, num_layers, 0, num_kv_heads, page_size, max_pages_per_seq, 1))
    return MD_ERR_INVALID_ARG;
  PageTopParams p;
  p.scores = scores;
  p.ids = ids;
  p.rows = num_layers * num_kv_heads;
  p.P_max = max_pages_per_seq;
  p.top = top_pages;
  p.first = first_pages;
  p.last = last_pages;
  p.n_seqs = batch;
  memcpy(p.n_pages, s.n_pages, sizeof(p.n_pages));
  return launch_page_top(p, (cudaStream_t)stream) == cudaSuccess ? MD_OK : MD_ERR_CUDA;
}

MD_API md_status md_attend_pages(const void *q, const void *pool, const int32_t *block_table, const int32_t *n_tokens,
                                 const int32_t *page_ids, void *out, float *mass, int batch, int num_layers,
                                 int num_q_heads, int num_kv_heads, int page_size, int max_pages_per_seq,
                                 int num_phys_pages, int top_pages, void *stream) {
  using namespace md;
  AttendPagesParams p;
  if (misaligned(q) || misaligned(pool) || !block_table || !page_ids || !out || ((uintptr_t)out & 7) || num_q_heads < 1 ||
      top_pages < 1 || (long long)top_pages * page_size > MD_MAX_TOP_TOKENS ||
      !page_set(p, block_table, n_tokens, batch, num_layers, num_q_heads, num_kv_heads, page_size, max_pages_per_seq,
                num_phys_pages))
    return MD_ERR_INVALID_ARG;
  p.q = (const uint16_t *)q;
  p.pool = (const uint16_t *)pool;
  p.out = (uint16_t *)out;
  p.ids = page_ids;
  p.mass = mass;
  p.mass_acc = nullptr;
  p.scale_log2 = (float)(1.4426950408889634 / sqrt((double)D));
  p.top = top_pages;
  return launch_attend_pages(p, (cudaStream_t)stream) == cudaSuccess ? MD_OK : MD_ERR_CUDA;
}
