/* Decode attention over a paged cache that the caller owns, in bf16 or in eight bits, under a
 * sliding window with first tokens that stay visible. */
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <math.h>

#include <algorithm>

#include "md_attn.cuh"

namespace md {

namespace {

constexpr int BLOCK = MD_SCALE_TOKENS;
static_assert(BLOCK == TILE, "a block is a matrix instruction's rows");
constexpr int STEP_BYTES = 8192;             // K and V of a step: 32 tokens of an e4m3 cache, 16 of a bf16 one
constexpr int PARTIAL = GP * D + 2 * GP;     // floats of a part of a row: O [8][128], exponents [8], sums [8]
constexpr int MAX_PARTIALS = MD_ATTEND_WORKSPACE / (PARTIAL * 4);
constexpr float SLACK = 10.f;                // log2 of the most that a weight may be above its base
constexpr float LIFT = 5.f;                  // log2 of the weight at the base (E4M3): f16 ends 2^-29 below it
constexpr float LOWER = 1.f / 32;            // 2^-LIFT, taken back by V's scales and the sums
constexpr int OS = D + 4;                    // padded row of a warp's O
static_assert(GP * OS * 4 <= STEP_BYTES, "a warp's O fits a stage");

struct AttendCacheParams : PageSet {
  const uint16_t *q;
  const void *pool;
  const float *scales;
  uint16_t *out;
  float *lse;                                // or null
  float *partials;                           // of rows that are split over units
  float scale_log2;                          // log2(e) / sqrt(D)
  long long limit_ns;                        // of the wait for a copy
  int lost_step;                             // of a warp, taken for one that did not land; -1: none
  int window, sinks;                         // window: INT_MAX for all
  int C;                                     // CTAs per unit
  int early;                                 // all CTAs run at once: their first pages go to L2 ahead of the wait
  int unit_start[MD_MAX_BATCH + 1];          // units of the sequences before, in the order that they are worked in
  int part_start[MD_MAX_BATCH];              // first partial of a sequence whose rows are split (in that order)
  uint8_t order[MD_MAX_BATCH];               // the sequence at each place of that order
};

/* The visible tokens of a sequence by blocks of 16: the first `head` blocks, and those from block
 * `tail` on; `blocks` in all. */
struct Visible {
  int w0, sinks;                             // tokens from w0 on, and the first `sinks`
  int head, tail, blocks;
};
__host__ __device__ __forceinline__ Visible visible(int n, int window, int sinks) {
  Visible v;
  v.w0 = n - window > 0 ? n - window : 0;
  v.sinks = sinks < v.w0 ? sinks : v.w0;
  v.head = (v.sinks + BLOCK - 1) / BLOCK;
  v.tail = v.w0 / BLOCK;
  if (v.tail <= v.head) v.head = v.tail = 0; // no block between them
  v.blocks = v.head + (n + BLOCK - 1) / BLOCK - v.tail;
  if (v.w0 == n) v.blocks = v.sinks ? (v.sinks + BLOCK - 1) / BLOCK : 0;
  return v;
}
/* Which of a block's tokens are visible. */
__device__ __forceinline__ uint32_t visible_mask(const Visible &v, int n, int tok) {
  auto below = [](int x) { return x <= 0 ? 0u : x >= BLOCK ? 0xffffu : (1u << x) - 1; };
  return below(n - tok) & (below(v.sinks - tok) | ~below(v.w0 - tok));
}

/* The maxima against which weights are taken: 0 where nothing but -inf was seen. */
__device__ __forceinline__ float max_base(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float inverse(float s) { return s > 0.f ? 1.f / s : s == 0.f ? 0.f : s; }   // NaN stays
__device__ __forceinline__ float logarithm(float base, float sum) {
  return sum == 0.f ? -INFINITY : 0.69314718f * (base + log2f(sum));
}

/* Bounded wait on an mbarrier phase. */
__device__ __noinline__ bool wait_copy(uint32_t bar, uint32_t parity, long long limit_ns) {
  const long long t0 = globaltimer();
  while (!mbar_try_wait(bar, parity))
    if (globaltimer() - t0 > limit_ns) return false;
  return true;
}

/* D(16x8, f32) = A(16x16, f16, row) * B(16x8, f16, col) + C */
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1, float c0, float c1, float c2, float c3) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%10,%11,%12,%13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
/* Two e4m3 codes (the lower and the upper 16 bits' two) as f16: exact. */
__device__ __forceinline__ uint32_t f16_lo(uint32_t c) {
  uint32_t r;
  asm("{.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;}" : "=r"(r) : "r"(c));
  return r;
}
__device__ __forceinline__ uint32_t f16_hi(uint32_t c) {
  uint32_t r;
  asm("{.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;}" : "=r"(r) : "r"(c));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 r;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(addr));
  return r;
}
__device__ __forceinline__ uint32_t word(const uint4 &x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }
/* Two 16x16 matrices of bytes, transposed: lane (g, t) gets columns g and g + 8 of each at rows 4t .. 4t + 3. */
__device__ __forceinline__ void ldmatrix_b8_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ void prefetch_l2(const void *p) {
  asm volatile("prefetch.global.L2 [%0];" ::"l"((uint64_t)__cvta_generic_to_global(p)) : "memory");
}
__device__ __forceinline__ void prefetch_l2_bulk(const void *p, uint32_t bytes) {     // multiples of 16
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"((uint64_t)__cvta_generic_to_global(p)), "r"(bytes)
               : "memory");
}

/* Sums over channels d .. d + 3 of bf16 V rows with finite weights, of which some came out NaN:
 * infinite where the row's visible tokens have infinite values of one sign and no NaN, as
 * every weight is above 0 (the two terms of a weight may be 0 or cancel, and their products with
 * an infinite value give NaN). */
__device__ __noinline__ float4 infinite_sums(const AttendCacheParams &p, int b, int l, int h, int d, float4 sums) {
  float *s = &sums.x;
  uint32_t seen = 0, open = 0;                       // 4 bits per channel: inf, -inf, NaN; those to be told
#pragma unroll
  for (int k = 0; k < 4; ++k) open |= (s[k] != s[k] ? 1u : 0u) << 4 * k;
  const int n = p.n_tokens[b];
  const Visible v = visible(n, p.window, p.sinks);
  for (int i = 0; i < v.blocks && open; ++i) {
    const int tok = (i < v.head ? i : i - v.head + v.tail) * BLOCK, pg = tok / p.ps;
    const int phys = p.block_table[(size_t)b * p.P_max + pg];
    if ((unsigned)phys >= (unsigned)p.P_phys) continue;
    const uint32_t mask = visible_mask(v, n, tok);
    const uint16_t *r = (const uint16_t *)p.pool +
                        (((((size_t)l * p.P_phys + phys) * p.Hkv + h) * 2 + 1) * p.ps + tok - pg * p.ps) * D + d;
#pragma unroll 8
    for (int t = 0; t < BLOCK; ++t) {
      if (!(mask >> t & 1)) continue;
      const uint2 w = *(const uint2 *)(r + t * D);
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

/* Four channels of a head of a row: divided by the sum, rounded, written. */
template <bool E4M3>
__device__ __forceinline__ void put_out(const AttendCacheParams &p, int b, int l, int h, int head, int d, float4 acc, float r) {
  if (!E4M3 && any_nan(acc) && r > 0.f) acc = infinite_sums(p, b, l, h, d, acc);
  uint16_t *dst = p.out + (((size_t)b * p.L + l) * p.Hq + h * p.G + head) * D + d;
  *(uint2 *)dst = make_uint2(pack_bf16(acc.x * r, acc.y * r), pack_bf16(acc.z * r, acc.w * r));
}

constexpr int ST = 2;                        // steps of a warp in flight
constexpr size_t attend_smem(int C, int warps) {
  return 1024 + (size_t)warps * ST * STEP_BYTES + (2 * warps * GP + 2 * GP) * 4 +
         (C > 1 ? (MAX_CLUSTER * GP * 2 + GP * D) * 4 : 0) + 128 + warps * ST * 8 + 8;
}

/* What works on a unit. */
enum Team { WARP, CTA, CLUSTER };

/* A unit is a (sequence, layer, KV head) row, or one of the equal parts of it; C CTAs of NW warps
 * per unit, a cluster, or, for many short rows, a warp.  The unit's blocks go to the warps in turn, a step at a time; a
 * warp copies its own steps by TMA (K and V rows, 128-byte swizzle), ST in flight, and computes
 *   S = K Q^T   rows are tokens, columns the group's heads
 *   O^T = V^T P^T  rows are channels, summed over the tokens.
 *
 * E4M3: codes become f16 on their way from shared memory into the fragments, exactly; the scales are
 * applied to the 32-bit results, K's to the scores and V's as a block's product is added to O.  K is
 * read 16 bytes of a row at a time (the summed channels are permuted alike in the queries), V by
 * transposed loads, four tokens of a channel per register.  Row g of the scores is token
 * t(g) = g ^ (4 if g is odd), row g + 8 token 8 + (t(g) ^ 4): with the swizzle, neither meets a bank
 * twice, and the weights lie where V's registers want them.
 *
 * The weights enter the product with V as two terms each, f16 for E4M3 (22 bits together) and bf16 for BF16
 * (16).  One f16 term (11 bits) was measured against two: 32 x 1,700 tokens in 36 layers 113.9 and 116.5 us,
 * 4 x 65,536 607 and 605, one layer of 131,071 tokens 14.9 and 15.8, 16 x 13,001 under a window of 4,096 9.3 and
 * 10.1.  It showed as 2^-12 of sum p |v| in outputs that cancel, so two are taken.
 *
 * The weights are taken against a base that follows the running maximum only when a score exceeds
 * it by SLACK: most steps then need no exchange between lanes and no rescaling. */
template <int NW, bool E4M3, Team TEAM>
__global__ void __launch_bounds__(32 * NW, NW == 4 ? 3 : 1)
    attend_cache_kernel(const __grid_constant__ AttendCacheParams p, const __grid_constant__ CUtensorMap tmap) {
  constexpr int NB = E4M3 ? 2 : 1;                   // blocks of a step
  constexpr int PER = 32 / NB;                       // steps whose blocks the lanes hold
  constexpr int BYTES = STEP_BYTES / NB;             // of a block
  constexpr int WARP_FLOATS = ST * STEP_BYTES / 4;
  constexpr bool ONE = TEAM != CLUSTER;
  extern __shared__ uint8_t smem_raw[];
  float *so = (float *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);   // [NW] the warps' stages, later their O [8][OS]
  float *zero = so + NW * WARP_FLOATS;               // 128 bytes of zeros
  float *sm = zero + 32;                             // [NW][8] exponents of the bases, then sums
  float *sl = sm + NW * GP;
  float *fin = sl + NW * GP;                         // [8] final bases, [8] 1 / sums
  float *xo = fin + 2 * GP;                          // [C][1024 / C] every CTA's part of this one's slice
  float *xml = xo + (ONE ? 0 : GP * D);              // [C][8][2]
  uint64_t *full = (uint64_t *)(xml + (ONE ? 0 : MAX_CLUSTER * GP * 2));    // [NW][ST]
  int *partial_at = (int *)(full + NW * ST);         // place of this unit among the partials
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int C = ONE ? 1 : p.C, unit = TEAM == WARP ? blockIdx.x * NW + warp : blockIdx.x / C, rank = ONE ? 0 : blockIdx.x - unit * C;
  const uint32_t ring = smem_u32(so) + warp * ST * STEP_BYTES, bars = smem_u32(full + warp * ST);
  if (lane < ST) {
    mbar_init(bars + lane * 8, NB);
    fence_barrier_init();
  }
  if (lane == 0) tma_prefetch_desc(&tmap);
  if (warp == 0) zero[lane] = 0.f;
  __syncthreads();
  if (TEAM == WARP && unit >= p.unit_start[p.n_seqs]) return;
  if (!ONE) cluster_arrive();                        // this CTA runs: the others may write its shared memory
  int place = 0;                                     // of the sequence: unit_start[place] <= unit < unit_start[place + 1]
  for (int hi = p.n_seqs; hi - place > 1;) {
    const int mid = (place + hi) >> 1;
    if (p.unit_start[mid] <= unit) place = mid;
    else hi = mid;
  }
  const int b = p.order[place], at_unit = unit - p.unit_start[place];
  if (TEAM != WARP && threadIdx.x == 0) *partial_at = p.part_start[place] + at_unit;
  const int lh = p.L * p.Hkv, parts = TEAM == WARP ? 1 : (p.unit_start[place + 1] - p.unit_start[place]) / lh;
  const int item = at_unit / parts, part = at_unit - item * parts;
  const int l = item / p.Hkv, h = item - l * p.Hkv;
  const int n_tok = p.n_tokens[b];
  const Visible vis = visible(n_tok, p.window, p.sinks);
  /* this unit's blocks, in whole steps but for the last */
  const int steps = (vis.blocks + NB - 1) / NB;
  const int s0 = (int)((long long)steps * part / parts), s1 = (int)((long long)steps * (part + 1) / parts);
  const int W = TEAM == WARP ? 1 : C * NW, w = TEAM == WARP ? 0 : rank * NW + warp;        // warps of the unit; this one takes steps s0 + w, s0 + w + W, ...
  const int nt = s1 - s0 > w ? (s1 - s0 - w + W - 1) / W : 0;
  const size_t q_row = ((size_t)b * p.L + l) * p.Hq + h * p.G;
  const uint64_t stream = policy_evict_first();
  const int per_page = p.ps / BLOCK, page_shift = per_page - 1;   // 1 or 2 blocks
  /* While the launch before ends: the pages of the first steps go into L2, by the table as it is
   * now.  Only where to look depends on it, so that an entry that is about to change costs a useless
   * copy; the table is read again behind the wait (and past L1 here, which would keep what it read).
   * One layer of 131,071 tokens 16.6 -> 15.9 us, 8 x 13,001 13.8 -> 13.1, 8 x 32,768 in bf16 in 4 layers
   * under a window of 1,000 9.4 -> 8.4; some launches lose: 1 x 20,000 8.5 -> 9.0, 32 x 1,700 8.4 -> 8.8.  Where CTAs
   * come in waves it gains nothing. */
  if (p.early) {
    const int i = (s0 + w + W * (lane / NB)) * NB + (lane & (NB - 1));
    if (lane / NB < min(ST, nt) && i < vis.blocks) {
      const int at = i < vis.head ? i : i - vis.head + vis.tail;
      const int page = ld_volatile(p.block_table + (size_t)b * p.P_max + (at >> page_shift));
      if ((unsigned)page < (unsigned)p.P_phys) {
        const size_t row = ((size_t)l * p.P_phys + page) * p.Hkv + h;
        const uint8_t *k_rows = (const uint8_t *)p.pool + (row * 2 * p.ps + (at & page_shift) * BLOCK) * (BYTES / 2 / BLOCK);
        prefetch_l2_bulk(k_rows, BYTES / 2);
        prefetch_l2_bulk(k_rows + (size_t)p.ps * (BYTES / 2 / BLOCK), BYTES / 2);
        if (E4M3) prefetch_l2(p.scales + (row * 2 << page_shift) + (at & page_shift));
      }
    }
  }
  pdl_wait();
  pdl_trigger();

  /* The lanes hold the blocks of a list of PER steps: lane i the block i % NB of its step i / NB.  Of
   * the list after it, the pages are looked up when a list begins, and the scales asked for in its middle. */
  auto block_of = [&](int list) {                    // the lane's block, or -1
    const int j = list + lane / NB, i = (s0 + w + W * j) * NB + (lane & (NB - 1));
    return j < nt && i < vis.blocks ? (i < vis.head ? i : i - vis.head + vis.tail) : -1;
  };
  auto look_up = [&](int list) {
    const int at = block_of(list);
    return at >= 0 ? p.block_table[(size_t)b * p.P_max + (at >> page_shift)] : -1;
  };
  struct Held {
    int row;                                         // of the tensor map
    uint32_t mask;                                   // visible tokens; in the upper half the block's place in its page
    float ks, vs;
  };
  auto open = [&](int list, int phys) {
    Held x = {0, 0, 0.f, 0.f};
    const int at = block_of(list);
    if (at >= 0 && (unsigned)phys < (unsigned)p.P_phys) {
      x.row = (l * p.P_phys + phys) * p.Hkv + h;
      x.mask = visible_mask(vis, n_tok, at * BLOCK) | (uint32_t)(at & page_shift) << 16;
      if (E4M3) {
        const float *s = p.scales + ((size_t)x.row * 2 << page_shift) + (at & page_shift);
        x.ks = s[0];
        x.vs = s[per_page];                          // not a use of it: the copy goes out first
      }
    }
    return x;
  };
  auto copy = [&](int j, const Held &x) {            // the lanes of step j
    const uint32_t bar = bars + (j & (ST - 1)) * 8, dst = ring + (j & (ST - 1)) * STEP_BYTES + (lane & (NB - 1)) * BYTES;
    if (x.mask) {
      const int sub = (x.mask >> 16) * BLOCK;
      mbar_arrive_expect_tx(bar, BYTES);
      tma_load_4d(dst, &tmap, 0, sub, 0, x.row, bar, stream);
      if (!E4M3) tma_load_4d(dst + BYTES / 2, &tmap, 64, sub, 0, x.row, bar, stream);
    } else {
      mbar_arrive(bar);
    }
  };
  int phys = look_up(0);
  Held held = open(0, phys), next = {0, 0, 0.f, 0.f};
  if (lane / NB < ST && lane / NB < nt) copy(lane / NB, held);

  uint32_t q[8][2];                                  // fragments of head g
  float qs[2] = {p.scale_log2, p.scale_log2};        // factors of the scores of heads 2t, 2t + 1
  if (E4M3) {                                        // channels 16 t + 4 i .., 64 + 16 t + 4 i ..
    uint32_t x[16];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 u = g < p.G ? *((const uint4 *)(p.q + (q_row + g) * D) + 8 * (i >> 1) + 2 * t + (i & 1)) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[4 * i + k] = word(u, k);
        most = max(most, max(word(u, k) << 16 & 0x7fff0000u, word(u, k) & 0x7fff0000u));
      }
    }
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
    /* f16 holds them relative to the largest: 2^-e x is below 2^15 */
    int e = (int)(most >> 23) - 127 - 14;
    e = most == 0 || most >= 0x7f800000u ? 0 : max(e, -126);
    const float down = __uint_as_float((127 - e) << 23), up = __uint_as_float((127 + e) << 23);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      q[i >> 1][i & 1] = pack_f16(__uint_as_float(x[i] << 16) * down, __uint_as_float(x[i] & 0xffff0000u) * down);
    qs[0] *= __shfl_sync(0xffffffffu, up, 8 * t);
    qs[1] *= __shfl_sync(0xffffffffu, up, 8 * t + 4);
  } else {                                           // channels 16 i + 2 t, + 1 and + 8, + 9
    const uint16_t *r = p.q + (q_row + g) * D + 2 * t;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      q[i][0] = g < p.G ? *(const uint32_t *)(r + 16 * i) : 0u;
      q[i][1] = g < p.G ? *(const uint32_t *)(r + 16 * i + 8) : 0u;
    }
  }
  /* tokens of rows g and g + 8 of the scores; the rows whose address this lane gives to ldmatrix */
  const int tok0 = E4M3 ? g ^ (g & 1) << 2 : g, tok1 = E4M3 ? 8 + (tok0 ^ 4) : g + 8;
  const int mi = lane >> 3, rr = lane & 7;
  const int pair = (lane & 15) >> 2 << 1 | (lane & 1), pair_tok = pair ^ (pair & 1) << 2;
  const int v_row = E4M3 ? (lane & 2 ? 8 + (pair_tok ^ 4) : pair_tok) : (mi >> 1) * 8 + rr;
  const uint32_t k_lane = E4M3 ? tok0 * 128 + ((t ^ tok0) << 4) : ((mi & 1) * 8 + rr) * 128 + (((mi >> 1) ^ rr) << 4);
  const uint32_t k_lane8 = tok1 * 128 + ((t ^ (tok1 & 7)) << 4);      // E4M3
  const uint32_t v_lane = (BLOCK + v_row) * 128 + (((E4M3 ? lane >> 4 : mi & 1) ^ (v_row & 7)) << 4);
  const uint32_t zeros = smem_u32(zero);
  float m[2] = {-INFINITY, -INFINITY}, z[2] = {0.f, 0.f}, o[8][4];
  float base[2] = {0.f, 0.f}, lim[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  bool landed = true;
  int k = 0;
  for (; k < nt; ++k) {
    if ((k & (PER / 2 - 1)) == 0) {
      if (k & (PER / 2)) {
        next = open((k & ~(PER - 1)) + PER, phys);
      } else {
        if (k) held = next;
        phys = look_up(k + PER);
      }
    }
    uint32_t seen[NB];
    float kscale[NB], vscale[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int from = (k & (PER - 1)) * NB + j;
      seen[j] = __shfl_sync(0xffffffffu, held.mask, from) & 0xffffu;
      if (E4M3) {
        kscale[j] = __shfl_sync(0xffffffffu, held.ks, from);
        vscale[j] = __shfl_sync(0xffffffffu, held.vs, from) * LOWER;
      }
    }
    const uint32_t st = ring + (k & (ST - 1)) * STEP_BYTES, bar = bars + (k & (ST - 1)) * 8, parity = k / ST & 1;
    landed = k != p.lost_step && (mbar_try_wait(bar, parity) || wait_copy(bar, parity, p.limit_ns));
    if (!__all_sync(0xffffffffu, landed)) {
      landed = false;
      break;
    }
    float c[NB][4];
    uint32_t v[NB][4][4];                            // E4M3: V's codes
    uint32_t v_at[NB];                               // rows of invisible tokens, whatever they hold: zeros
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
      const uint32_t kb = st + j * BYTES + k_lane;
      v_at[j] = seen[j] >> v_row & 1 ? st + j * BYTES + v_lane : zeros;
      if (E4M3) {
        const uint32_t kb8 = st + j * BYTES + k_lane8;
        const uint4 a = lds128(kb), a8 = lds128(kb8), e = lds128(kb ^ 64), e8 = lds128(kb8 ^ 64);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          mma_f16(x, f16_lo(word(a, i)), f16_lo(word(a8, i)), f16_hi(word(a, i)), f16_hi(word(a8, i)), q[i][0], q[i][1], x[0],
                  x[1], x[2], x[3]);
          mma_f16(y, f16_lo(word(e, i)), f16_lo(word(e8, i)), f16_hi(word(e, i)), f16_hi(word(e8, i)), q[4 + i][0],
                  q[4 + i][1], y[0], y[1], y[2], y[3]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) ldmatrix_b8_trans(v_at[j] ^ i << 5, v[j][i]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint32_t a0, a1, a2, a3;
          ldmatrix_x4((kb ^ (i & 3) << 5) + (i >> 2) * (BYTES / 2), a0, a1, a2, a3);
          mma_bf16(i & 1 ? y : x, a0, a1, a2, a3, q[i][0], q[i][1]);
        }
      }
      /* heads 2t, 2t + 1 of tokens tok0 (0, 1) and tok1 (2, 3) */
      const float f0 = E4M3 ? qs[0] * kscale[j] : qs[0], f1 = E4M3 ? qs[1] * kscale[j] : qs[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) c[j][i] = (x[i] + y[i]) * (i & 1 ? f1 : f0);
      if (seen[j] != 0xffffu) {
        const bool in0 = seen[j] >> tok0 & 1, in1 = seen[j] >> tok1 & 1;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!(i < 2 ? in0 : in1)) c[j][i] = -INFINITY;
      }
    }
    float mx[2] = {fmaxf(c[0][0], c[0][2]), fmaxf(c[0][1], c[0][3])};
#pragma unroll
    for (int j = 1; j < NB; ++j) {
      mx[0] = fmaxf(mx[0], fmaxf(c[j][0], c[j][2]));
      mx[1] = fmaxf(mx[1], fmaxf(c[j][1], c[j][3]));
    }
    if (__any_sync(0xffffffffu, mx[0] > lim[0] || mx[1] > lim[1])) {
#pragma unroll
      for (int s = 4; s < 32; s <<= 1)
#pragma unroll
        for (int i = 0; i < 2; ++i) mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], s));
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float last = m[i];                     // -inf: nothing to rescale
        m[i] = fmaxf(m[i], mx[i]);
        const float alpha = ex2(last - max_base(m[i]));
        base[i] = max_base(m[i]) - (E4M3 ? LIFT : 0.f);
        lim[i] = m[i] + SLACK;
        z[i] *= alpha;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          o[j][i] *= alpha;
          o[j][2 + i] *= alpha;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = ex2(c[j][i] - base[i & 1]);
      z[0] += x[0] + x[2];
      z[1] += x[1] + x[3];
      if (E4M3) {
        /* two f16 terms: the nearest, and the nearest to what is left, which is exact */
        const uint32_t u0 = pack_f16(x[0], x[1]), u1 = pack_f16(x[2], x[3]);
        const float2 h0 = __half22float2(*(const __half2 *)&u0), h1 = __half22float2(*(const __half2 *)&u1);
        const uint32_t b0 = movmatrix_trans(u0), b1 = movmatrix_trans(u1);
        const uint32_t r0 = movmatrix_trans(pack_f16(x[0] - h0.x, x[1] - h0.y)), r1 = movmatrix_trans(pack_f16(x[2] - h1.x, x[3] - h1.y));
#pragma unroll
        for (int i = 0; i < 8; ++i) {                // channels 16 i + g, + 8
          const uint32_t c0 = v[j][i >> 1][2 * (i & 1)], c8 = v[j][i >> 1][2 * (i & 1) + 1];
          const uint32_t a0 = f16_lo(c0), a1 = f16_lo(c8), a2 = f16_hi(c0), a3 = f16_hi(c8);
          float d[4];
          mma_f16(d, a0, a1, a2, a3, r0, r1, 0.f, 0.f, 0.f, 0.f);
          mma_f16(d, a0, a1, a2, a3, b0, b1, d[0], d[1], d[2], d[3]);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][e] = fmaf(d[e], vscale[j], o[i][e]);
        }
      } else {
        uint32_t hi[2], lo[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t u = pack_bf16(x[2 * i], x[2 * i + 1]);
          hi[i] = movmatrix_trans(u);
          lo[i] = movmatrix_trans(
              pack_bf16(x[2 * i] - __uint_as_float(u << 16), x[2 * i + 1] - __uint_as_float(u & 0xffff0000u)));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {                // channels 16 i + g, + 8
          uint32_t a0, a1, a2, a3;
          ldmatrix_x4_trans((v_at[j] ^ (i & 3) << 5) + (v_at[j] == zeros ? 0 : (i >> 2) * (BYTES / 2)), a0, a1, a2, a3);
          mma_bf16(o[i], a0, a1, a2, a3, hi[0], hi[1]);
          mma_bf16(o[i], a0, a1, a2, a3, lo[0], lo[1]);
        }
      }
    }
    __syncwarp();
    const int j = k + ST;
    if (j < nt && lane / NB == (j & (PER - 1))) {    // refill the stage: its reads come before the copy
      fence_proxy_async_smem();
      copy(j, (k ^ j) & PER ? next : held);
    }
  }
  if (!landed) {                                     // what is in flight must land before the stages are reused
    for (int j = k; j < min(k + ST, nt); ++j) wait_copy(bars + (j & (ST - 1)) * 8, j / ST & 1, DRAIN_LIMIT_NS);
    z[0] = z[1] = NAN;
  }
#pragma unroll
  for (int s = 4; s < 32; s <<= 1)
#pragma unroll
    for (int i = 0; i < 2; ++i) z[i] += __shfl_xor_sync(0xffffffffu, z[i], s);
  if (g == 0)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sm[warp * GP + 2 * t + i] = m[i];
      sl[warp * GP + 2 * t + i] = E4M3 ? z[i] * LOWER : z[i];
    }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      so[warp * WARP_FLOATS + (2 * t + (e & 1)) * OS + 16 * i + g + 8 * (e >> 1)] = o[i][e];
    }
  const size_t lse_row = ((size_t)b * p.L + l) * p.Hq + h * p.G;
  if (TEAM == WARP) {
    __syncwarp();
    for (int head = 0; head < p.G; ++head) {
      const float sum = sl[warp * GP + head];
      const float4 e = *(const float4 *)&so[warp * WARP_FLOATS + head * OS + 4 * lane];
      put_out<E4M3>(p, b, l, h, head, 4 * lane, e, inverse(sum));
      if (p.lse && lane == 0) p.lse[lse_row + head] = logarithm(max_base(sm[warp * GP + head]), sum);
    }
    return;
  }
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
    const float to = max_base(top[i]);
    sum[i] = 0.f;
    acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int y = 0; y < NW; ++y) {
      const float f = ex2(sm[y * GP + head] - to);
      const float4 e = *(const float4 *)&so[y * WARP_FLOATS + head * OS + 4 * lane];
      sum[i] += f * sl[y * GP + head];
      acc[i].x += f * e.x;
      acc[i].y += f * e.y;
      acc[i].z += f * e.z;
      acc[i].w += f * e.w;
    }
  }
  float *partial = p.partials + (size_t)*partial_at * PARTIAL;   // where parts > 1
  if (ONE) {
#pragma unroll
    for (int i = 0; i < GP / NW; ++i) {
      const int head = warp + i * NW;
      if (parts > 1) {
        *(float4 *)(partial + head * D + 4 * lane) = acc[i];
        if (lane == 0) {
          partial[GP * D + head] = top[i];
          partial[GP * D + GP + head] = sum[i];
        }
      } else if (head < p.G) {
        put_out<E4M3>(p, b, l, h, head, 4 * lane, acc[i], inverse(sum[i]));
        if (p.lse && lane == 0) p.lse[lse_row + head] = logarithm(max_base(top[i]), sum[i]);
      }
    }
    return;
  }
  cluster_wait();                                    // every CTA runs
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
    const float to = max_base(most);
    for (int y = 0; y < C; ++y) s += ex2(xml[(y * GP + head) * 2] - to) * xml[(y * GP + head) * 2 + 1];
    fin[head] = to;
    fin[GP + head] = inverse(s);
    if (rank == 0) {
      if (parts > 1) {
        partial[GP * D + head] = most;
        partial[GP * D + GP + head] = s;
      } else if (p.lse && head < p.G) {
        p.lse[lse_row + head] = logarithm(to, s);
      }
    }
  }
  __syncthreads();
  for (int e = threadIdx.x * 4; e < slice; e += 32 * NW * 4) {
    const int at_e = rank * slice + e, head = at_e / D;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < C; ++i) {
      const float f = ex2(xml[(i * GP + head) * 2] - fin[head]);
      const float4 x = *(const float4 *)&xo[i * slice + e];
      y.x += f * x.x;
      y.y += f * x.y;
      y.z += f * x.z;
      y.w += f * x.w;
    }
    if (parts > 1)
      *(float4 *)(partial + at_e) = y;
    else if (head < p.G)
      put_out<E4M3>(p, b, l, h, head, at_e - head * D, y, fin[GP + head]);
  }
}

/* The parts of split rows together: a block per row and pair of heads, four warps per head that take
 * its parts in turn, four channels per lane.  Latency bounds it: the parts' sums are asked for before
 * their bases are known. */
struct JoinParams : AttendCacheParams {
  uint8_t split[MD_MAX_BATCH];               // places of the sequences whose rows are split
};
template <bool E4M3>
__global__ void __launch_bounds__(256) attend_join_kernel(const __grid_constant__ JoinParams p) {
  constexpr int AHEAD = 8;                   // parts of a warp under way
  __shared__ float4 so[8][32];
  __shared__ float sl[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, turn = warp & 3;
  const int item = blockIdx.x >> 2, head = (blockIdx.x & 3) * 2 + (warp >> 2);
  const int place = p.split[blockIdx.y], b = p.order[place];
  const int lh = p.L * p.Hkv, parts = (p.unit_start[place + 1] - p.unit_start[place]) / lh;
  const int l = item / p.Hkv, h = item - l * p.Hkv;
  const float *from = p.partials + (size_t)(p.part_start[place] + item * parts) * PARTIAL;
  pdl_wait();
  pdl_trigger();
  float4 x[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (turn + 4 * i < parts) x[i] = *(const float4 *)(from + (size_t)(turn + 4 * i) * PARTIAL + head * D + 4 * lane);
  float top = -INFINITY;
  for (int y = lane; y < parts; y += 32) top = fmaxf(top, from[(size_t)y * PARTIAL + GP * D + head]);
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
  const float base = max_base(top);
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = 0.f;
  for (int y0 = turn; y0 < parts; y0 += 4 * AHEAD) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int y = y0 + 4 * i;
      if (y >= parts) break;
      const float *r = from + (size_t)y * PARTIAL;
      const float f = ex2(r[GP * D + head] - base);
      if (y0 != turn) x[i] = *(const float4 *)(r + head * D + 4 * lane);
      sum += f * r[GP * D + GP + head];
      acc.x += f * x[i].x;
      acc.y += f * x[i].y;
      acc.z += f * x[i].z;
      acc.w += f * x[i].w;
    }
  }
  so[warp][lane] = acc;
  if (lane == 0) sl[warp] = sum;
  __syncthreads();
  if (turn || head >= p.G) return;
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    const float4 e = so[warp + i][lane];
    sum += sl[warp + i];
    acc.x += e.x;
    acc.y += e.y;
    acc.z += e.z;
    acc.w += e.w;
  }
  put_out<E4M3>(p, b, l, h, head, 4 * lane, acc, inverse(sum));
  if (p.lse && lane == 0) p.lse[((size_t)b * p.L + l) * p.Hq + h * p.G + head] = logarithm(base, sum);
}

struct Form {
  Team team = CTA;
  int C = 1, warps = 4, unit = 0;            // CTAs per unit, warps per CTA, most steps of a unit
  bool waves = false;                        // more CTAs than run at once
};

/* How many CTAs and warps per unit, and how many steps a unit has at most: the estimate of the
 * launch's time that is least.  A warp's step takes `step` us with 4, 8 or 12 warps on its SM; a CTA
 * of 4 warps shares its SM with two others, one of 8 warps has it alone.  Where all CTAs run at once, the
 * longest one's steps and the bytes at the copy rate both bound the time (their 4-norm: near each
 * other, neither hides the other); with several waves, the CTAs' summed time and the bytes, and a
 * last wave of the CTAs that are left, which are shorter ones: then the longest rows go first (16
 * sequences of 2,000 to 4,001 tokens in 36 layers 134.1 -> 131.2 us).
 *   The constants were fitted to 91 launches timed on a GB300 in up to 45 forms each (1 to 128
 * sequences, 1 to 36 layers, 1 to 8 KV heads, 100 to 131,071 tokens, both types, a third of them ragged or
 * under a window), and a warp per row was weighed against a CTA of 4 in 86 more (72 to 18,432 rows, most of them
 * short), while the weights over E4M3 were one f16 term; with two a launch takes up to 9% longer.
 * All 177 were then timed again, each in its 25 fastest forms: the one taken is 0.9% slower than the
 * best on average, more than 5% in 12 of them, 14% at worst (512 rows of 150 tokens in bf16: CTAs 11.3 us, warps
 * 9.9); profiles/attend_cache_forms.csv has them.  Some forms, us: one sequence of 131,071 tokens, 2 KV heads: 16 parts,
 * each a cluster of 4 CTAs of 8 warps, which is taken, 15.9, of 8 of 4 warps 15.9, one part of 16 CTAs of 8 37; 448
 * tokens: 4 CTAs of 4 warps, taken, 4.1, 8 4.3, one of 8 warps 4.7; 32 x 1,700 in 36 layers: one CTA of 4 warps, taken,
 * 118, two 146, one of 8 152; 4 x 65,536 in 36 layers: one of 8, taken, 615, two of 8 623, one of 4 659.
 *   A warp per row is taken for many short rows, whose CTAs would mostly start and end: 64 rows of 40
 * tokens in 8 KV heads 6.9 -> 4.4 us, 36 windows of 16 in 16 layers and 4 heads 21.1 -> 9.8, 64 sequences of
 * 120 to 600 in 36 layers and 2 heads 82 -> 69. */
Form attend_form(AttendCacheParams &p, bool e4m3, bool workspace) {
  constexpr float SMS = 152.f;
  const int NB = e4m3 ? 2 : 1, lh = p.L * p.Hkv;
  int steps[MD_MAX_BATCH], most = 0;
  long long total = 0;
  for (int b = 0; b < p.n_seqs; ++b) {
    steps[b] = (visible(p.n_tokens[b], p.window, p.sinks).blocks + NB - 1) / NB;
    most = std::max(most, steps[b]);
    total += (long long)steps[b] * lh;
  }
  const float step4 = e4m3 ? 0.657f : 0.489f, step8 = e4m3 ? 0.813f : 0.628f, step12 = e4m3 ? 1.218f : 0.908f;
  const float bytes = (float)total * (STEP_BYTES * 0.978f / 6.69e6f);   // us at the copy rate
  auto norm = [](float x, float y) { return sqrtf(sqrtf(x * x * x * x + y * y * y * y)); };
  Form best;
  best.unit = std::max(most, 1);
  float least = INFINITY;
  for (const int parts : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
    const int unit = std::max((most + parts - 1) / parts, 1);
    if (parts > 1 && (!workspace || unit < 8)) break;
    long long units = 0, partials = 0;
    for (int b = 0; b < p.n_seqs; ++b) {
      const int n = std::max((steps[b] + unit - 1) / unit, 1);
      units += n;
      if (n > 1) partials += n;
    }
    if (partials * lh > MAX_PARTIALS) break;
    auto consider = [&](Team team, int C, int warps) {
      const int team_warps = team == WARP ? 1 : C * warps;
      /* a cluster of 8 or 16 CTAs leaves parts of the chip unused */
      const float part = warps == 4 ? (C <= 2 ? 1.f : C == 4 ? 0.95f : C == 8 ? 0.93f : 0.74f)
                                    : (C <= 2 ? 1.f : C == 4 ? 0.94f : C == 8 ? 0.8f : 0.6f);
      const float N = team == WARP ? ceilf((float)units * lh / warps) : (float)units * lh * C;
      const float slots = SMS * part * (warps == 4 ? 3 : 1);
      const float longest = (float)((unit + team_warps - 1) / team_warps);
      const float start = 2.65f + (team == WARP ? 0.25f : 0.f) + (C > 1 ? 0.82f : 0.f) + (C == 16 ? 0.187f : 0.f) + (warps == 8 ? 0.139f : 0.f);
      /* of a warp, where n CTAs run */
      auto step = [&](float n) { return warps == 8 || (n > SMS * part && n <= 2 * SMS * part) ? step8 : n <= SMS * part ? step4 : step12; };
      float t;
      if (N <= slots) {
        t = start + norm(longest * step(N), bytes) + 0.0019f * N;
      } else {
        const float steps_each = (float)total / (N * warps) + 0.5f;
        const float cta = start + 1.316f + 0.701f * log2f((float)C) + steps_each * step(slots);
        const float waves = floorf(N / slots), left = N - waves * slots;
        const float last = 0.6f * longest + 0.4f * std::min(longest, steps_each);
        t = start + norm(waves * cta, bytes * (1.f - left / N)) + std::max(0.533f * last * step(left), bytes * left / N);
        t = std::max(t, start + 1.316f + 0.81f * longest * step(slots));
      }
      if (team == WARP) t *= 1.1f;                                       // a warp whose row ends early idles
      if (parts > 1) t += 1.791f + 0.0217f * parts;
      if (t < least) {
        least = t;
        best.team = team;
        best.C = C;
        best.warps = warps;
        best.unit = unit;
        best.waves = N > slots;
      }
    };
    for (int warps = 4; warps <= 8; warps += 4)
      for (int C = 1; C <= MAX_CLUSTER; C *= 2) {
        if (C * warps > 4 && C * warps >= 2 * unit) break;             // half of them would have no step
        consider(C > 1 ? CLUSTER : CTA, C, warps);
      }
    if (parts == 1) consider(WARP, 1, 4);
  }
  auto parts_of = [&](int b) { return std::max((steps[b] + best.unit - 1) / best.unit, 1); };
  uint32_t key[MD_MAX_BATCH];                // steps of a unit, then the sequence
  for (int b = 0; b < p.n_seqs; ++b) key[b] = (uint32_t)(steps[b] / parts_of(b)) << 8 | (uint32_t)b;
  if (best.waves) std::sort(key, key + p.n_seqs, [](uint32_t x, uint32_t y) { return x > y; });
  p.unit_start[0] = 0;
  int partials = 0;
  for (int i = 0; i < p.n_seqs; ++i) {
    const int b = key[i] & 255, n = parts_of(b) * lh;
    p.order[i] = (uint8_t)b;
    p.part_start[i] = partials;
    if (n > lh) partials += n;
    p.unit_start[i + 1] = p.unit_start[i] + n;
  }
  return best;
}

template <int NW, bool E4M3, Team TEAM>
cudaError_t launch_attend(const AttendCacheParams &p, const CUtensorMap &tmap, cudaStream_t s) {
  constexpr int which = ATTR_ATTEND_CACHE + (E4M3 ? 1 : 0) + 2 * TEAM + (NW == 8 ? 6 : 0);
  constexpr bool ONE = TEAM != CLUSTER;
  const auto kernel = attend_cache_kernel<NW, E4M3, TEAM>;
  const cudaError_t e = once_per_device<which>([&] {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)attend_smem(ONE ? 1 : MAX_CLUSTER, NW));
    return e != cudaSuccess || ONE ? e : cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(TEAM == WARP ? (p.unit_start[p.n_seqs] + NW - 1) / NW : p.unit_start[p.n_seqs] * p.C));
  cfg.blockDim = dim3(32 * NW);
  cfg.dynamicSmemBytes = attend_smem(p.C, NW);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.C;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ONE ? 1 : 2;
  return cudaLaunchKernelEx(&cfg, kernel, p, tmap);
}

/* Blocks of K and V rows of a pool in eight bits: 128 bytes x 16 rows x (K, V), swizzled. */
bool encode_block_map(void *encode, CUtensorMap *m, const void *pool, size_t items, int ps) {
  const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)ps, 2, (cuuint64_t)items};
  const cuuint64_t strides[3] = {(cuuint64_t)D, (cuuint64_t)D * ps, (cuuint64_t)D * ps * 2};
  const cuuint32_t box[4] = {(cuuint32_t)D, BLOCK, 2, 1}, one[4] = {1, 1, 1, 1};
  return ((decltype(&cuTensorMapEncodeTiled))encode)(
             m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, (void *)pool, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool E4M3>
cudaError_t run(AttendCacheParams &p, const CUtensorMap &tmap, bool workspace, cudaStream_t s) {
  const Form f = attend_form(p, E4M3, workspace);
  p.C = f.C;
  p.early = !f.waves;
  cudaError_t e = f.team == WARP    ? launch_attend<4, E4M3, WARP>(p, tmap, s)
                  : f.team == CTA ? (f.warps == 8 ? launch_attend<8, E4M3, CTA>(p, tmap, s) : launch_attend<4, E4M3, CTA>(p, tmap, s))
                  : f.warps == 8  ? launch_attend<8, E4M3, CLUSTER>(p, tmap, s)
                                  : launch_attend<4, E4M3, CLUSTER>(p, tmap, s);
  const int lh = p.L * p.Hkv;
  JoinParams j;
  int split = 0;
  for (int b = 0; b < p.n_seqs; ++b)
    if (p.unit_start[b + 1] - p.unit_start[b] > lh) j.split[split++] = (uint8_t)b;
  if (e == cudaSuccess && split) {
    (AttendCacheParams &)j = p;
    e = launch_pdl(attend_join_kernel<E4M3>, dim3(4 * lh, split), 256, 0, s, j);
  }
  return e;
}

/* A wait for a copy gives up after limit_ns; lost_step: as above, for tests. */
md_status attend_cache(const md_attend_cache_args *args, long long limit_ns = 2000000000LL, int lost_step = -1) {
  if (!args) return MD_ERR_INVALID_ARG;
  const md_attend_cache_args &a = *args;
  AttendCacheParams p;
  auto aligned = [](const void *x, size_t to) { return x && ((uintptr_t)x & (to - 1)) == 0; };
  const bool e4m3 = a.type == MD_TYPE_E4M3;
  if ((!e4m3 && a.type != MD_TYPE_BF16) || a.window < -1 || a.sinks < 0 || a.num_q_heads < 1 || !aligned(a.q_dev, 16) ||
      !aligned(a.pool_dev, 16) || (e4m3 && !aligned(a.scales_dev, 4)) || !aligned(a.block_table_dev, 4) ||
      !aligned(a.out_dev, 8) || ((uintptr_t)a.lse_dev & 3) ||
      !page_set(p, a.block_table_dev, a.n_tokens_host, a.batch, a.num_layers, a.num_q_heads, a.num_kv_heads, a.page_size,
                a.max_pages_per_seq, a.num_phys_pages))
    return MD_ERR_INVALID_ARG;
  if (a.workspace_dev && ((uintptr_t)a.workspace_dev & 15 || a.workspace_bytes < MD_ATTEND_WORKSPACE))
    return MD_ERR_WORKSPACE;
  p.q = (const uint16_t *)a.q_dev;
  p.pool = a.pool_dev;
  p.scales = a.scales_dev;
  p.out = (uint16_t *)a.out_dev;
  p.lse = a.lse_dev;
  p.partials = (float *)a.workspace_dev;
  p.scale_log2 = (float)(1.4426950408889634 / sqrt((double)D));
  p.limit_ns = limit_ns;
  p.lost_step = lost_step;
  p.window = a.window < 0 ? INT32_MAX : a.window;
  p.sinks = a.sinks;
  void *encode = tile_encoder();
  CUtensorMap tmap;
  const size_t items = (size_t)a.num_layers * a.num_phys_pages * a.num_kv_heads;
  if (!encode || !(e4m3 ? encode_block_map(encode, &tmap, a.pool_dev, items, a.page_size)
                        : encode_tile_map(encode, &tmap, (void *)a.pool_dev, items * 2 * a.page_size, a.page_size)))
    return MD_ERR_CUDA;
  const cudaStream_t s = (cudaStream_t)a.stream;
  const bool workspace = a.workspace_dev != nullptr;
  return (e4m3 ? run<true>(p, tmap, workspace, s) : run<false>(p, tmap, workspace, s)) == cudaSuccess ? MD_OK : MD_ERR_CUDA;
}

}  // namespace

}  // namespace md

extern "C" __attribute__((visibility("default"))) md_status md_attend_cache(const md_attend_cache_args *args) {
  return md::attend_cache(args);
}
