/* Decode attention over the pages that a cheap score selects: bounds of a page's
 * keys, the bound of its logits, the selection, and the attention over it. */
#include <cuda_bf16.h>

#include <math.h>
#include <string.h>

#include <algorithm>
#include <atomic>

#include "md_attn.cuh"

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

/* A warp per 16 pages of a (sequence, layer, KV head): the pages are an MMA's rows,
 * the query heads its columns, and lo and hi side by side the summed dimension,
 * against the queries' negative and positive parts.
 *
 * The sum is left in the instructions' 32-bit accumulators: against 64 bits it is off by
 * 1.6e-7 (rms, relative), three times what separate operations would be.
 *
 * HBM bounds it, given registers for all of a tile's loads at once (64 a thread):
 * 2.1 M pages (1.08 GB of bounds) 161 us, 99% of the copy rate; 171 with 80 registers
 * and fewer warps, 180 with 54, where the loads went out in two parts, 167 with the
 * pages that are not there kept in a register, which spilled one. */
__global__ void __launch_bounds__(256, 4) page_scores_kernel(const __grid_constant__ PageScoresParams p, int tiles) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int lh = p.L * p.Hkv;
  const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);   // tiles: of the longest sequence
  const int row = (int)(unit / tiles), tile = (int)(unit - (long long)row * tiles);
  if (row >= p.n_seqs * lh) return;
  const int b = row / lh, l = row % lh / p.Hkv, h = row % p.Hkv;
  const int P = p.n_pages[b], p0 = tile * 16 + g, p1 = p0 + 8;
  if (tile * 16 >= P) return;
  uint32_t q[16];
  load_q(p.q + (((size_t)b * p.L + l) * p.Hq + h * p.G) * D, p.G, g, t, q);
  const int i0 = page_id(p, b, p0), i1 = page_id(p, b, p1);
  const uint4 *s0 = (const uint4 *)(p.bounds + (((size_t)l * p.P_phys + (i0 < 0 ? 0 : i0)) * p.Hkv + h) * 2 * D) + t;
  const uint4 *s1 = (const uint4 *)(p.bounds + (((size_t)l * p.P_phys + (i1 < 0 ? 0 : i1)) * p.Hkv + h) * 2 * D) + t;
  const uint32_t nan2 = 0x7FFF7FFFu;             // a page without tokens: told from a NaN key at the end
  const uint4 none = make_uint4(nan2, nan2, nan2, nan2);
  uint4 x[8], y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {                // 0..3: lo, 4..7: hi
    x[j] = i0 >= 0 ? s0[4 * j] : none;
    y[j] = i1 >= 0 ? s1[4 * j] : none;
  }
  float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = j < 4 ? min2(q[4 * (j & 3) + k], 0u) : max2(q[4 * (j & 3) + k], 0u);
    mma_bf16(c, x[j].x, y[j].x, x[j].y, y[j].y, w[0], w[1]);
    mma_bf16(c, x[j].z, y[j].z, x[j].w, y[j].w, w[2], w[3]);
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
  if (t == 0 && p0 < P) dst[p0] = m0 == m0 || page_id(p, b, p0) >= 0 ? m0 * p.scale : -INFINITY;
  if (t == 0 && p1 < P) dst[p1] = m1 == m1 || page_id(p, b, p1) >= 0 ? m1 * p.scale : -INFINITY;
}

/* ---------------------------------------------------------------- top --- */
/* fp32 -> uint32 in the same order; NaN above all, the zeros equal */
__device__ __forceinline__ uint32_t score_key(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

/* A block per row, KEYS keys per thread in registers.  A histogram over the range
 * that the row's keys span (not over fixed bits: the scores of a row lie close
 * together) finds the bin with the k-th largest, then one over that bin, until a bin is
 * taken whole or holds equal keys: two rounds for most rows.  The pages that are
 * taken become bits, and one scan over the words of bits gives all places.
 *
 * Latency bounds it: barriers and round trips through shared memory; with several blocks
 * per SM also the atomics, one per key and round.  2 rows of 2,048
 * pages 4.0 us, 576 rows of 4,096 9.6 us.  With keys in shared memory and a second pass
 * over them for the places 5.6 and 15.7; with eight-bit digits 7.3 and 24.3. */
constexpr int BINS = 2048;

/* Sum of a over the threads before this one; every thread calls it. */
__device__ __forceinline__ int scan_before(int a, int warps, int *warp_sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = a;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += u;
  }
  if (lane == 31) warp_sum[warp] = x;
  __syncthreads();
  return x - a + __reduce_add_sync(0xffffffffu, lane < warp ? warp_sum[lane] : 0);
}

template <int threads, int KEYS>
__global__ void __launch_bounds__(threads) page_top_kernel(const __grid_constant__ PageTopParams p) {
  constexpr int warps = threads / 32;
  __shared__ int hist[BINS], warp_sum[32];
  __shared__ uint32_t warp_lo[32], warp_hi[32], above[warps * KEYS], equal[warps * KEYS];
  __shared__ int s_bin, s_left, s_in;
  pdl_wait();
  pdl_trigger();
  const size_t row = (size_t)blockIdx.y * gridDim.x + blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int P = p.n_pages[blockIdx.y];
  int32_t *out = p.ids + row * p.top;
  if (P <= p.top) {
    for (int i = tid; i < p.top; i += threads) out[i] = i < P ? i : -1;
    return;
  }
  const int n = P - p.first - p.last;          // pages to choose from
  int left = p.top - p.first - p.last;         // how many
  const float *sc = p.scores + row * p.P_max + p.first;
  for (int i = tid; i < p.first; i += threads) out[i] = i;
  for (int i = tid; i < p.last; i += threads) out[p.top - p.last + i] = P - p.last + i;
  if (left == 0) return;
  uint32_t k[KEYS], lo = 0xffffffffu, hi = 0;
#pragma unroll
  for (int i = 0; i < KEYS; ++i) {
    const int at = tid + i * threads;
    k[i] = at < n ? score_key(sc[at]) : 0u;    // 0: the key of no score
  }
#pragma unroll
  for (int i = 0; i < KEYS; ++i) {
    lo = min(lo, k[i] - 1);                    // past the end: 0xffffffff
    hi = max(hi, k[i]);
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (lane == 0) {
    warp_lo[warp] = lo;
    warp_hi[warp] = hi;
  }
#pragma unroll
  for (int i = 0; i < BINS; i += threads) hist[i + tid] = 0;
  __syncthreads();
  lo = __reduce_min_sync(0xffffffffu, lane < warps ? warp_lo[lane] : 0xffffffffu) + 1;
  hi = __reduce_max_sync(0xffffffffu, lane < warps ? warp_hi[lane] : 0u);
  /* keys above hi are taken, and `left` of those in [lo, hi] */
  while (true) {
    const uint32_t span = hi - lo;
    const int bits = 32 - __clz(span), shift = bits > 11 ? bits - 11 : 0;
#pragma unroll
    for (int i = 0; i < KEYS; ++i)
      if (k[i] - lo <= span) atomicAdd(&hist[(k[i] - lo) >> shift], 1);
    __syncthreads();
    constexpr int each = BINS / threads;       // bins per thread, from the top down
    int sum = 0;
#pragma unroll
    for (int i = 0; i < each; ++i) sum += hist[BINS - 1 - tid * each - i];
    int before = scan_before(sum, warps, warp_sum);
    if (before < left && left <= before + sum) {
      int bin = BINS - 1 - tid * each;
      while (before + hist[bin] < left) before += hist[bin--];
      s_bin = bin;
      s_left = left - before;
      s_in = hist[bin];
    }
    __syncthreads();
    left = s_left;
    lo += (uint32_t)s_bin << shift;
    hi = lo + min(hi - lo, (1u << shift) - 1);
    if (s_in == left || shift == 0) break;
#pragma unroll
    for (int i = 0; i < BINS; i += threads) hist[i + tid] = 0;
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < KEYS; ++i) {             // word w: pages 32 w ..
    const unsigned gt = __ballot_sync(0xffffffffu, k[i] > hi), eq = __ballot_sync(0xffffffffu, k[i] - lo <= hi - lo);
    if (lane == 0) {
      above[warp + i * warps] = gt;
      equal[warp + i * warps] = eq;
    }
  }
  __syncthreads();
  const bool mine = tid < KEYS * warps;        // a word per thread
  const uint32_t gt = mine ? above[tid] : 0u, eq = mine ? equal[tid] : 0u;
  const int at = scan_before(__popc(gt) | __popc(eq) << 16, warps, warp_sum);   // at most 16,384 of each
  int a = at & 0xffff, e = at >> 16;
  for (uint32_t any = gt | eq; any; any &= any - 1) {
    const uint32_t bit = any & (0u - any);
    const bool is_gt = gt & bit;
    if (is_gt || e < left) out[p.first + a + min(e, left)] = p.first + 32 * tid + __ffs(bit) - 1;
    a += is_gt;
    e += !is_gt;
  }
}

/* ------------------------------------------------------------- attend --- */
/* A cluster of C CTAs of NW warps per (sequence, layer, KV head).  The tiles of
 * a list, 16 tokens of a page each, go to the cluster's warps in turn; a warp
 * copies its own tiles by TMA (K and V rows, 64-channel halves, 128-byte
 * swizzle), one or two in flight, and computes
 *   S = K Q^T   rows are tokens, columns the group's heads
 *   O^T = V^T P^T  rows are channels, summed over the tokens.
 *
 * The weights enter the product as two bf16 terms each (16 bits of them): one
 * term would add about as much error as the output's own rounding.
 * They are taken against a base that follows the running maximum only when a
 * score exceeds it by SLACK: most tiles then need no exchange between lanes and
 * no rescaling.
 *
 * With an infinite value the terms' products cancel or are 0 times it, and the sum is NaN
 * (infinite_sums).
 *
 * The masses need the scores again with the final maxima and sums.  A row of one CTA
 * keeps them in tensor memory, four columns per tile in its warp's lanes: the shared
 * memory is left to the tiles, and up to four CTAs share an SM where their scores would
 * leave room for one (4 x 65,536 tokens, 36 layers: 105 -> 96 us).  A cluster keeps them
 * in shared memory: a row's tiles are spread over more warps there, and no CTA waits for
 * columns while another waits for it.  Each of its CTAs pushes its maxima and sums, and
 * its part of the others' slices of O, into the others' shared memory; after one cluster
 * barrier each has all it needs.
 *
 * A copy that does not land within the limit makes its row NaN (and is reported
 * in the status words, where there are any). */
constexpr int SCORE_BYTES = TILE * GP * 4;   // one tile's
constexpr int TILE_BYTES = 2 * TILE * D * 2; // 16 K rows and 16 V rows
constexpr int STAGES = 2;                    // most tiles in flight per warp
constexpr float SLACK = 10.f;                // log2 of the most that a weight may be
constexpr int OS = D + 4;                    // padded row of a warp's O
constexpr int MAX_ATTEND_SMEM = 227 * 1024;
static_assert(GP * OS * 4 <= TILE_BYTES, "a warp's O fits a stage");
constexpr size_t attend_smem(int C, int warps, int stages, int warp_tiles) {
  return 1024 + (size_t)warps * (stages * TILE_BYTES + warp_tiles * (4 + (C > 1 ? SCORE_BYTES : 0))) + 2 * warps * GP * 4 +
         2 * GP * 4 + (C > 1 ? (MAX_CLUSTER * GP * 2 + GP * D) * 4 : 0) + warps * STAGES * 8 + 8;
}

/* Columns of tensor memory that hold the scores of a CTA's warps (of C = 1): a power of
 * two, 32 at least; above TM_COLUMNS there is no room.  Warps w and w + 4 share lanes. */
constexpr int TM_COLUMNS = 512;
constexpr int attend_columns(int warps, int warp_tiles) {
  int n = 32;
  while (n < 4 * warp_tiles * (warps / 4)) n *= 2;
  return n;
}

struct AttendParams : AttendPagesParams {
  int C, stages;       // CTAs per row; tiles in flight per warp
  int warp_tiles;      // most tiles of a warp whose scores are kept
  int columns;         // of tensor memory (C = 1), where scores are kept
};

/* Bounded wait on an mbarrier phase. */
__device__ __noinline__ bool wait_copy(uint32_t bar, uint32_t parity, long long limit_ns) {
  const long long t0 = globaltimer();
  while (!mbar_try_wait(bar, parity))
    if (globaltimer() - t0 > limit_ns) return false;
  return true;
}

/* The maxima against which weights are taken: 0 where nothing but -inf was seen. */
__device__ __forceinline__ float max_base(float m) { return m == -INFINITY ? 0.f : m; }

/* Sums over channels d .. d + 3 of V rows with finite weights, of which some came out
 * NaN: infinite where the row's tokens have infinite values of one sign and no NaN, as
 * every weight is above 0.  A pass over those channels, for such sums only, up to the
 * page that shows all of them to be NaN (the first one, if all values are).  With
 * infinite values a call takes about 1 us more per page of a list, 4 x 65,536 tokens of
 * nothing else in 36 layers 767 us instead of 97. */
__device__ __noinline__ float4 infinite_sums(const AttendParams &p, int row, int b, int l, int h, int d, float4 sums) {
  float *s = &sums.x;
  uint32_t seen = 0, open = 0;                       // 4 bits per channel: inf, -inf, NaN; those to be told
#pragma unroll
  for (int k = 0; k < 4; ++k) open |= (s[k] != s[k] ? 1u : 0u) << 4 * k;
  for (int e = 0; e < p.top && open; ++e) {
    const int pg = p.ids[(size_t)row * p.top + e], phys = page_id(p, b, pg);
    if (phys < 0) continue;
    const int n = page_tokens(p, b, pg);
    const uint16_t *v = p.pool + ((((size_t)(p.l0 + l) * p.P_phys + phys) * p.Hkv + h) * 2 + 1) * p.ps * D + d;
#pragma unroll 8
    for (int i = 0; i < n; ++i) {
      const uint2 w = *(const uint2 *)(v + i * D);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t x = (k < 2 ? w.x : w.y) >> 16 * (k & 1);
        if ((x & 0x7f80u) == 0x7f80u) seen |= (x & 0x7fu ? 4u : x & 0x8000u ? 2u : 1u) << 4 * k;
      }
    }
    open &= ~(seen >> 2 | (seen & seen >> 1));
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (open >> 4 * k & 1u && seen >> 4 * k & 3u) s[k] = seen >> 4 * k & 1u ? INFINITY : -INFINITY;
  return sums;
}
__device__ __forceinline__ bool any_nan(float4 x) { return isnan(x.x + x.y) || isnan(x.z + x.w); }

/* ---- tensor memory ---- */
__device__ __forceinline__ void tm_alloc(uint32_t smem, int columns) {      // a whole warp
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tm_free(uint32_t at, int columns) {         // the same warp
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void tm_before_barrier() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tm_after_barrier() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tm_store4(uint32_t at, const float (&x)[4]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(__float_as_uint(x[0])),
               "r"(__float_as_uint(x[1])), "r"(__float_as_uint(x[2])), "r"(__float_as_uint(x[3]))
               : "memory");
}
__device__ __forceinline__ void tm_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_load8(uint32_t at, float (&x)[8]) {
  uint32_t u[8];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
      : "r"(at)
      : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(u[i]);
}

/* ONE: C is 1.  TM: scores are kept, in tensor memory.  With and without masses are two
 * kernels: in one, CTAs without masses, which never came to tm_alloc, ran as if there were
 * one per SM, and their calls took up to 3 times as long. */
template <int NW, bool ONE, bool TM>
__global__ void __launch_bounds__(32 * NW)
    attend_pages_kernel(const __grid_constant__ AttendParams p, const __grid_constant__ CUtensorMap tmap) {
  extern __shared__ uint8_t smem_raw[];
  const int stages = p.stages, WARP_FLOATS = stages * TILE_BYTES / 4;
  float *so = (float *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);   // [NW] the warps' stages, later their O [8][OS]
  float *sc = so + NW * WARP_FLOATS;                 // [NW][warp_tiles][16][8] scores (not ONE)
  float *sm = sc + (ONE ? 0 : NW * p.warp_tiles * TILE * GP);   // [NW][8] maxima, then sums
  float *sl = sm + NW * GP;
  float *fin = sl + NW * GP;                         // [8] final maxima, [8] 1 / sums
  float *xo = fin + 2 * GP;                          // [C][1024 / C] every CTA's part of this one's slice
  float *xml = xo + (ONE ? 0 : GP * D);              // [C][8][2]
  uint64_t *full = (uint64_t *)(xml + (ONE ? 0 : MAX_CLUSTER * GP * 2));   // [NW][STAGES]
  uint32_t *columns = (uint32_t *)(full + NW * STAGES);   // address of the tensor memory (ONE)
  int *sv = (int *)(columns + 2);                    // [NW][warp_tiles] tokens per tile
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int mi = lane >> 3, rr = lane & 7;           // ldmatrix: matrix and row of this lane's address
  const int C = ONE ? 1 : p.C, row = blockIdx.x / C, rank = blockIdx.x - row * C;
  const uint32_t ring = smem_u32(so) + warp * stages * TILE_BYTES, bars = smem_u32(full + warp * STAGES);
  if (lane < STAGES) {
    mbar_init(bars + lane * 8, 1);
    fence_barrier_init();
  }
  if (lane == 0) tma_prefetch_desc(&tmap);
  __syncwarp();
  if (!ONE) cluster_arrive();                        // this CTA runs: the others may write its shared memory
  const int lh = p.L * p.Hkv;
  const int b = row / lh, l = row % lh / p.Hkv, h = row % p.Hkv;
  const int shift = p.ps / TILE - 1, tiles = p.top << shift;   // tiles per page: 1 or 2
  const size_t q_row = ((size_t)b * p.L + l) * p.Hq + h * p.G;
  const int W = C * NW, w = rank * NW + warp;        // warps of the row; this one takes tiles w, w + W, ...
  const int nt = tiles > w ? (tiles - w + W - 1) / W : 0;
  float *wsc = sc + warp * p.warp_tiles * TILE * GP;
  int *wsv = sv + warp * p.warp_tiles;
  const bool masses = ONE ? TM : p.mass || p.mass_acc;
  const uint64_t stream = policy_evict_first();
  pdl_wait();
  /* Columns are taken after the launch before has freed its own, and before the next one may
   * start: whoever waits for columns holds up none of those who have them. */
  if (TM) {
    if (warp == 0) tm_alloc(smem_u32(columns), p.columns);
  } else {
    pdl_trigger();
  }
  /* tile n0 + lane of this warp: its page's row of the tensor map, its rows' offset there, its tokens */
  auto tile_info = [&](int n0, int &at, int &sub, int &valid) {
    at = sub = valid = 0;
    if (n0 + lane < nt) {
      const int tile = w + W * (n0 + lane), pg = p.ids[(size_t)row * p.top + (tile >> shift)];
      const int phys = page_id(p, b, pg);
      sub = (tile & shift) * TILE;
      if (phys >= 0) {
        valid = max(0, min(TILE, page_tokens(p, b, pg) - sub));
        at = ((p.l0 + l) * p.P_phys + phys) * p.Hkv + h;
      }
    }
  };
  auto copy_tile = [&](int stage, int at, int sub) {
    const uint32_t dst = ring + stage * TILE_BYTES, bar = bars + stage * 8;
    mbar_arrive_expect_tx(bar, TILE_BYTES);
    tma_load_4d(dst, &tmap, 0, sub, 0, at, bar, stream);
    tma_load_4d(dst + TILE_BYTES / 2, &tmap, 64, sub, 0, at, bar, stream);
  };
  int at, sub, valid;
  tile_info(0, at, sub, valid);
  uint32_t q[8][2];                                  // head g, channels 16 kk + 2t, + 1 and + 8, + 9
  {
    const uint16_t *r = p.q + (q_row + g) * D + 2 * t;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      q[kk][0] = g < p.G ? *(const uint32_t *)(r + 16 * kk) : 0u;
      q[kk][1] = g < p.G ? *(const uint32_t *)(r + 16 * kk + 8) : 0u;
    }
  }
  float m[2] = {-INFINITY, -INFINITY}, z[2] = {0.f, 0.f}, o[8][4];
  float base[2] = {0.f, 0.f}, lim[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  int done = 0, issued = 0;                          // tiles of this warp, across the lists of 32
  unsigned todo, ahead;                              // of a list: tiles to compute, to copy
  bool landed = true;
  auto begin = [&](int n0) {                         // the first tiles of a list, a lane each
    if (masses && n0 + lane < nt) wsv[n0 + lane] = valid;
    todo = ahead = __ballot_sync(0xffffffffu, valid > 0);
    const int i = __popc(todo & ((1u << lane) - 1));
    if (valid > 0 && i < stages) copy_tile((done + i) & (stages - 1), at, sub);
    issued += min(__popc(todo), stages);
    for (int k = 0; k < stages; ++k) ahead &= ahead - 1;
  };
  begin(0);
  uint32_t tm = 0;                                   // this warp's columns, four per tile
  if (TM) {
    tm_before_barrier();
    __syncthreads();
    tm_after_barrier();
    pdl_trigger();
    tm = *columns + (warp >> 2) * (p.columns / (NW / 4)) + ((warp & 3) << 21);   // lanes 32 (warp % 4) ..
  }
  for (int n0 = 0; n0 < nt; n0 += 32) {
    if (n0) {
      tile_info(n0, at, sub, valid);
      fence_proxy_async_smem();                      // behind the reads of the tiles before
      begin(n0);
    }
    for (; todo; todo &= todo - 1, ++done) {
      const int n = __ffs(todo) - 1, have = __shfl_sync(0xffffffffu, valid, n);
      const int stage = done & (stages - 1);       // stages: 1 or 2
      const uint32_t st = ring + stage * TILE_BYTES, bar = bars + stage * 8, parity = done >> (stages - 1) & 1;
      landed = done != p.lost_tile && (mbar_try_wait(bar, parity) || wait_copy(bar, parity, p.limit_ns));
      if (!__all_sync(0xffffffffu, landed)) {
        landed = false;
        break;
      }
      float c[4] = {0.f, 0.f, 0.f, 0.f}, c2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) {
        uint32_t a0, a1, a2, a3;
        ldmatrix_x4(swz<TILE>(st, (mi & 1) * 8 + rr, kk * 16 + (mi >> 1) * 8), a0, a1, a2, a3);
        mma_bf16(kk & 1 ? c2 : c, a0, a1, a2, a3, q[kk][0], q[kk][1]);
      }
      /* token g, heads 2t, 2t + 1; token g + 8 */
#pragma unroll
      for (int i = 0; i < 4; ++i)
        c[i] = g + 8 * (i >> 1) < have && 2 * t + (i & 1) < p.G ? (c[i] + c2[i]) * p.scale_log2 : -INFINITY;
      if (TM) {
        tm_store4(tm + (n0 + n) * 4, c);
      } else if (masses) {
        float *d = wsc + (n0 + n) * TILE * GP + g * GP + 2 * t;
        *(float2 *)d = make_float2(c[0], c[1]);
        *(float2 *)(d + 8 * GP) = make_float2(c[2], c[3]);
      }
      float mx[2] = {fmaxf(c[0], c[2]), fmaxf(c[1], c[3])};
      if (__any_sync(0xffffffffu, mx[0] > lim[0] || mx[1] > lim[1])) {
#pragma unroll
        for (int s = 4; s < 32; s <<= 1)
#pragma unroll
          for (int i = 0; i < 2; ++i) mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], s));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float last = m[i];                   // -inf: nothing to rescale
          m[i] = fmaxf(m[i], mx[i]);
          base[i] = max_base(m[i]);
          const float alpha = ex2(last - base[i]);
          lim[i] = m[i] + SLACK;
          z[i] *= alpha;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            o[j][i] *= alpha;
            o[j][2 + i] *= alpha;
          }
        }
      }
      uint32_t hi[2], lo[2];
      {
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = ex2(c[j] - base[j & 1]);
        z[0] += x[0] + x[2];
        z[1] += x[1] + x[3];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t u = pack_bf16(x[2 * j], x[2 * j + 1]);
          hi[j] = movmatrix_trans(u);
          lo[j] = movmatrix_trans(
              pack_bf16(x[2 * j] - __uint_as_float(u << 16), x[2 * j + 1] - __uint_as_float(u & 0xffff0000u)));
        }
      }
      /* V rows past the tile's tokens, whatever they hold: the last one again */
      const int vrow = TILE + min((mi >> 1) * 8 + rr, have - 1);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t a0, a1, a2, a3;
        ldmatrix_x4_trans(swz<TILE>(st, vrow, i * 16 + (mi & 1) * 8), a0, a1, a2, a3);
        mma_bf16(o[i], a0, a1, a2, a3, hi[0], hi[1]);
        mma_bf16(o[i], a0, a1, a2, a3, lo[0], lo[1]);
      }
      __syncwarp();
      if (ahead) {                                   // refill the stage: its reads come before the copy
        const int k = __ffs(ahead) - 1;
        const int at_k = __shfl_sync(0xffffffffu, at, k), sub_k = __shfl_sync(0xffffffffu, sub, k);
        if (lane == 0) {
          fence_proxy_async_smem();
          copy_tile(stage, at_k, sub_k);
        }
        ++issued;
        ahead &= ahead - 1;
      }
    }
    if (!landed) {                                   // the lists that are left have no tokens
      for (int n = n0 + 32 + lane; masses && n < nt; n += 32) wsv[n] = 0;
      break;
    }
  }
  if (!landed) {                                     // what is in flight must land before the stages are reused
    for (; done < issued; ++done) wait_copy(bars + (done & (stages - 1)) * 8, done >> (stages - 1) & 1, DRAIN_LIMIT_NS);
    z[0] = z[1] = NAN;
    if (p.status && lane == 0) {
      atomicCAS(&p.status[ST_CODE], 0, (int)MD_ERR_DEVICE_TIMEOUT);
      atomicExch(&p.status[ST_ABORT], 1);
    }
  }
#pragma unroll
  for (int s = 4; s < 32; s <<= 1)
#pragma unroll
    for (int i = 0; i < 2; ++i) z[i] += __shfl_xor_sync(0xffffffffu, z[i], s);
  if (g == 0)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sm[warp * GP + 2 * t + i] = m[i];
      sl[warp * GP + 2 * t + i] = z[i];
    }
#pragma unroll
  for (int i = 0; i < 8; ++i)                 // channels 16 i + g and + 8
#pragma unroll
    for (int j = 0; j < 4; ++j) so[warp * WARP_FLOATS + (2 * t + (j & 1)) * OS + 16 * i + g + 8 * (j >> 1)] = o[i][j];
  __syncthreads();
  /* the CTA's sums: 4 channels of a head per thread, 8 / NW heads per warp */
  const int slice = GP * D / C;
  float4 acc[GP / NW];
  float top[GP / NW], sum[GP / NW];
#pragma unroll
  for (int i = 0; i < GP / NW; ++i) {
    const int head = warp + i * NW;
    top[i] = -INFINITY;
#pragma unroll
    for (int y = 0; y < NW; ++y) top[i] = fmaxf(top[i], sm[y * GP + head]);
    const float base = max_base(top[i]);
    sum[i] = 0.f;
    acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int y = 0; y < NW; ++y) {
      const float f = ex2(sm[y * GP + head] - base);
      const float4 e = *(const float4 *)&so[y * WARP_FLOATS + head * OS + 4 * lane];
      sum[i] += f * sl[y * GP + head];
      acc[i].x += f * e.x;
      acc[i].y += f * e.y;
      acc[i].z += f * e.z;
      acc[i].w += f * e.w;
    }
  }
  auto inverse = [](float s) { return s > 0.f ? 1.f / s : s == 0.f ? 0.f : s; };   // no token: zeros; NaN stays
  if (ONE) {
#pragma unroll
    for (int i = 0; i < GP / NW; ++i) {
      const int head = warp + i * NW;
      const float r = inverse(sum[i]);
      if (any_nan(acc[i]) && r > 0.f) acc[i] = infinite_sums(p, row, b, l, h, 4 * lane, acc[i]);
      if (head < p.G)
        *(uint2 *)(p.out + (q_row + head) * D + 4 * lane) =
            make_uint2(pack_bf16(acc[i].x * r, acc[i].y * r), pack_bf16(acc[i].z * r, acc[i].w * r));
      if (lane == 0) {
        fin[head] = max_base(top[i]);
        fin[GP + head] = head < p.G ? r : 0.f;
      }
    }
    if (!masses) return;
    __syncthreads();
  } else {
    cluster_wait();                           // every CTA runs
#pragma unroll
    for (int i = 0; i < GP / NW; ++i) {
      const int head = warp + i * NW, e = head * D + 4 * lane, to = e / slice;
      st_cluster_v4(cluster_map(smem_u32(xo + rank * slice + e - to * slice), to), acc[i].x, acc[i].y, acc[i].z, acc[i].w);
      if (lane < C) st_cluster_v2(cluster_map(smem_u32(xml + (rank * GP + head) * 2), lane), top[i], sum[i]);
    }
    cluster_arrive();
    cluster_wait();
    if (threadIdx.x < GP) {
      const int head = threadIdx.x;
      float most = -INFINITY, s = 0.f;
      for (int y = 0; y < C; ++y) most = fmaxf(most, xml[(y * GP + head) * 2]);
      most = max_base(most);
      for (int y = 0; y < C; ++y) s += ex2(xml[(y * GP + head) * 2] - most) * xml[(y * GP + head) * 2 + 1];
      fin[head] = most;
      fin[GP + head] = head < p.G ? inverse(s) : 0.f;
    }
    __syncthreads();
    for (int e = threadIdx.x * 4; e < slice; e += 32 * NW * 4) {
      const int at_e = rank * slice + e, head = at_e / D;
      const float r = fin[GP + head];
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i = 0; i < C; ++i) {
        const float f = ex2(xml[(i * GP + head) * 2] - fin[head]);
        const float4 x = *(const float4 *)&xo[i * slice + e];
        y.x += f * x.x;
        y.y += f * x.y;
        y.z += f * x.z;
        y.w += f * x.w;
      }
      if (any_nan(y) && r > 0.f) y = infinite_sums(p, row, b, l, h, at_e - head * D, y);
      if (head < p.G)
        *(uint2 *)(p.out + q_row * D + at_e) =
            make_uint2(pack_bf16(y.x * r, y.y * r), pack_bf16(y.z * r, y.w * r));
    }
    if (!masses) return;
  }
  /* the masses of this warp's tiles, two at a time: a lane per token */
  const uint64_t keep = policy_evict_last();
  auto put = [&](int n, int tok, bool in, float x) {
    const int tile = w + W * n;
    if (p.mass) p.mass[((size_t)row * tiles + tile) * TILE + tok] = x;
    if (p.mass_acc && in)
      red_add_u64_hint(p.mass_acc + (size_t)page_id(p, b, p.ids[(size_t)row * p.top + (tile >> shift)]) * p.ps +
                           (tile & shift) * TILE + tok,
                       __float2ull_rn(x * MASS_SCALE), keep);
  };
  if constexpr (ONE) {
    const float m0 = fin[2 * t], m1 = fin[2 * t + 1], z0 = fin[GP + 2 * t], z1 = fin[GP + 2 * t + 1];
    tm_store_wait();
    for (int n0 = 0; n0 < nt; n0 += 2) {
      float c[8], x[4];                              // tokens g, g + 8 of tile n0, of the next: heads 2t, 2t + 1
      tm_load8(tm + n0 * 4, c);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = ex2(c[2 * i] - m0) * z0 + ex2(c[2 * i + 1] - m1) * z1;
        x[i] += __shfl_xor_sync(0xffffffffu, x[i], 1);
        x[i] += __shfl_xor_sync(0xffffffffu, x[i], 2);
      }
      const int n = n0 + (t >> 1), tok = g + 8 * (t & 1);
      if (n < nt) {
        const bool in = tok < wsv[n];
        put(n, tok, in, in ? (t & 2 ? (t & 1 ? x[3] : x[2]) : (t & 1 ? x[1] : x[0])) : 0.f);
      }
      __syncwarp();
    }
    tm_before_barrier();
    __syncthreads();
    tm_after_barrier();
    if (warp == 0) tm_free(*columns, p.columns);
  } else {
    float fm[GP], fz[GP];
#pragma unroll
    for (int i = 0; i < GP; ++i) {
      fm[i] = fin[i];
      fz[i] = fin[GP + i];
    }
    const int tok = lane & 15;
#pragma unroll 2
    for (int n0 = 0; n0 < nt; n0 += 2) {
      const int n = n0 + (lane >> 4);
      if (n >= nt) continue;
      const int have = wsv[n];
      const float4 *s = (const float4 *)(wsc + (n * TILE + tok) * GP);
      float x = 0.f;
      if (tok < have) {
        const float4 u = s[0], v = s[1];
        x = (ex2(u.x - fm[0]) * fz[0] + ex2(u.y - fm[1]) * fz[1]) + (ex2(u.z - fm[2]) * fz[2] + ex2(u.w - fm[3]) * fz[3]);
        x += (ex2(v.x - fm[4]) * fz[4] + ex2(v.y - fm[5]) * fz[5]) + (ex2(v.z - fm[6]) * fz[6] + ex2(v.w - fm[7]) * fz[7]);
      }
      put(n, tok, tok < have, x);
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
  const long long rows = (long long)p.n_seqs * p.L * p.Hkv, tiles = (most + 15) / 16;
  if (tiles == 0) return cudaSuccess;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((rows * tiles + 7) / 8));
  cfg.blockDim = dim3(256);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, page_scores_kernel, p, (int)tiles);
}

cudaError_t launch_page_top(const PageTopParams &p, cudaStream_t s) {
  int most = 0;
  for (int b = 0; b < p.n_seqs; ++b) most = p.n_pages[b] > most ? p.n_pages[b] : most;
  static_assert(MD_MAX_CHUNKS * MD_MAX_CHUNK_TOKENS / 16 <= 16 * 1024, "the longest row has its keys");
  const dim3 grid(p.rows, p.n_seqs);
  return most <= 1024   ? launch_pdl(page_top_kernel<512, 2>, grid, 512, 0, s, p)
         : most <= 2048 ? launch_pdl(page_top_kernel<512, 4>, grid, 512, 0, s, p)
         : most <= 4096 ? launch_pdl(page_top_kernel<512, 8>, grid, 512, 0, s, p)
         : most <= 8192 ? launch_pdl(page_top_kernel<1024, 8>, grid, 1024, 0, s, p)
                        : launch_pdl(page_top_kernel<1024, 16>, grid, 1024, 0, s, p);
}

namespace {

template <int NW, bool ONE, bool TM>
cudaError_t launch_attend(const AttendParams &p, const CUtensorMap &tmap, cudaStream_t s) {
  constexpr int which = (NW == 8 ? ATTR_ATTEND_8 : ATTR_ATTEND_4) + (TM ? 2 : ONE ? 1 : 0);
  const cudaError_t e = once_per_device<which>([] {
    const auto kernel = attend_pages_kernel<NW, ONE, TM>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_ATTEND_SMEM);
    return e != cudaSuccess || ONE ? e : cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.n_seqs * p.L * p.Hkv * p.C));
  cfg.blockDim = dim3(32 * NW);
  cfg.dynamicSmemBytes = attend_smem(p.C, NW, p.stages, p.warp_tiles);
  /* no more CTAs on an SM than there are columns for: none waits for them */
  if (TM)
    cfg.dynamicSmemBytes = std::max<size_t>(cfg.dynamicSmemBytes, 228 * 1024 / (TM_COLUMNS / p.columns + 1));
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.C;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ONE ? 1 : 2;
  return cudaLaunchKernelEx(&cfg, attend_pages_kernel<NW, ONE, TM>, p, tmap);
}

}  // namespace

namespace {

struct AttendForm {
  int C = 0, warps = 0, stages = 0;
};

/* How many CTAs and warps per row, and how many tiles in flight per warp.  cta: the
 * time of one CTA in us, n tiles of its busiest warp at 0.72 or, with two in flight,
 * 0.42; slots: CTAs that run at once (a cluster of 8 or 16 leaves parts of the chip
 * unused, the more so with one CTA per SM).  Of the forms whose CTAs all run at once the
 * shortest; if there is none, the one with the least CTA time per slot.  (What a
 * launch takes beyond that, HBM for one, is the same in all forms.)
 *   The constants were fitted to 115 launches timed on a GB300 in up to 20 forms each (1
 * to 64 sequences, 1 to 36 layers, 2 to 600 tiles per list, 2 to 7,200 rows, up to
 * 110 us at the copy rate).  Of 150 launches of 15 us and more at the copy rate, those
 * with masses take 1.7% longer than with the best form of each on average, 23% at worst;
 * all 2.3%, and 57% at worst: rows of a few tiles under lists of hundreds, without masses.
 * Some forms: 2 rows of 64 tiles 4.6 us with 16 x 4 warps, 8.4 with 8; 64 rows of 48, 8.3
 * with 4 x 4 and 8.5 with 8 or 2 x 8; 288 rows of 256, 96 with 8 or 4, 106 with 2 x 8.
 *   The scores' room counts whether masses are wanted or not: the split, and with it the
 * rounding of a result, does not depend on it.  The tiles in flight do. */
AttendForm attend_form(const AttendPagesParams &p) {
  constexpr float SMS = 152.f;
  const int tpp = p.ps / TILE, listed = p.top * tpp;
  int T = 1;
  for (int b = 0; b < p.n_seqs; ++b) T = std::max(T, std::min(p.n_pages[b], p.top) * tpp);
  const float rows = (float)p.n_seqs * p.L * p.Hkv;
  auto cost = [&](int C, int warps, int stages, bool scores) {
    const int W = C * warps, warp_tiles = scores ? (listed + W - 1) / W : 0;
    const size_t smem = attend_smem(C, warps, stages, warp_tiles);
    const int columns = C == 1 ? attend_columns(warps, warp_tiles) : 32;
    if (smem > MAX_ATTEND_SMEM || columns > TM_COLUMNS) return INFINITY;
    int per_sm = 1;                          // by shared memory, tensor memory and registers
    while (per_sm < std::min(16 / warps, TM_COLUMNS / columns) && (per_sm + 1) * (smem + 1024) <= 228 * 1024) ++per_sm;
    const float part = C <= 2 ? 1.f : per_sm > 1 ? (C == 4 ? 0.97f : C == 8 ? 0.93f : 0.72f)
                                                 : (C == 4 ? 0.94f : C == 8 ? 0.78f : 0.6f);
    const float slots = per_sm * SMS * part, N = rows * C;
    const float cta = 4.f + (C > 1 ? 0.73f : 0.f) + (C == 16 ? 0.13f : 0.f) + (warps == 8 ? 0.21f : 0.f) +
                      (float)((T + W - 1) / W) * (stages == 1 ? 0.72f : 0.42f);
    return N <= slots ? cta + 0.0021f * N : 1e6f + N / slots * cta + 0.0012f * N;
  };
  AttendForm best;
  float least = INFINITY;
  for (int C = 1; C <= MAX_CLUSTER; C *= 2)
    for (int warps = 4; warps <= 8; warps += 4)
      for (int stages = 1; stages <= STAGES; ++stages) {
        if (C * warps > 2 * listed && C * warps > 8) continue;
        const float x = cost(C, warps, stages, true);
        if (x < least) {
          least = x;
          best.C = C;
          best.warps = warps;
          best.stages = stages;
        }
      }
  if (best.C && !p.mass && !p.mass_acc)
    best.stages = cost(best.C, best.warps, 2, false) < cost(best.C, best.warps, 1, false) ? 2 : 1;
  return best;
}

}  // namespace

cudaError_t launch_attend_pages(const AttendPagesParams &base, const CUtensorMap &tmap, cudaStream_t s) {
  AttendParams p;
  (AttendPagesParams &)p = base;
  const AttendForm f = attend_form(base);
  if (f.C == 0) return cudaErrorInvalidConfiguration;   // MD_MAX_TOP_TOKENS fit 16 CTAs of 4 warps
  static_assert(attend_smem(MAX_CLUSTER, 4, 1, MD_MAX_TOP_TOKENS / TILE / (4 * MAX_CLUSTER)) <= MAX_ATTEND_SMEM,
                "the longest list has a form");
  const int W = f.C * f.warps;
  p.C = f.C;
  p.stages = f.stages;
  p.warp_tiles = p.mass || p.mass_acc ? (p.top * (p.ps / TILE) + W - 1) / W : 0;
  p.columns = attend_columns(f.warps, p.warp_tiles);
  auto launch = [&](auto eight, auto four) { return f.warps == 8 ? eight(p, tmap, s) : four(p, tmap, s); };
  return f.C > 1         ? launch(launch_attend<8, false, false>, launch_attend<4, false, false>)
         : p.warp_tiles  ? launch(launch_attend<8, true, true>, launch_attend<4, true, true>)
                         : launch(launch_attend<8, true, false>, launch_attend<4, true, false>);
}

bool page_set(PageSet &p, const int32_t *block_table, const int32_t *n_tokens, int batch, int L, int Hq, int Hkv, int ps,
              int P_max, int P_phys) {
  if (!n_tokens || batch < 1 || batch > MD_MAX_BATCH || L < 1 || L > 255 || Hkv < 1 || (ps != 16 && ps != 32) ||
      P_max < 1 || P_phys < 1 || (long long)P_max * ps > (long long)MD_MAX_CHUNKS * MD_MAX_CHUNK_TOKENS)
    return false;
  if (Hq && (Hq < Hkv || Hq % Hkv || Hq / Hkv > MD_MAX_GROUP)) return false;
  if ((long long)L * P_phys * Hkv * 2 * ps >= (1LL << 31) || (long long)batch * L * Hkv >= (1LL << 27)) return false;
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

void *tile_encoder() {
  static std::atomic<void *> known{nullptr};
  void *fn = known.load();
  if (!fn) {
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      return nullptr;
    known.store(fn);
  }
  return fn;
}

namespace {

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
  p.l0 = 0;
  p.status = nullptr;
  p.limit_ns = 2000000000LL;
  p.lost_tile = -1;
  void *encode = tile_encoder();
  CUtensorMap tmap;
  const size_t rows = (size_t)num_layers * num_phys_pages * num_kv_heads * 2 * page_size;
  if (!encode || !encode_tile_map(encode, &tmap, (void *)pool, rows, page_size)) return MD_ERR_CUDA;
  return launch_attend_pages(p, tmap, (cudaStream_t)stream) == cudaSuccess ? MD_OK : MD_ERR_CUDA;
}
