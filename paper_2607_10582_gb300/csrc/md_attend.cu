/* Decode attention over a paged cache that the caller owns, in bf16 or in eight bits, under a
 * sliding window with first tokens that stay visible. */
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <math.h>

#include "md_internal.h"
#include "md_ptx.cuh"

namespace md {

namespace {

constexpr int BLOCK = MD_SCALE_TOKENS;

struct AttendCacheParams : PageSet {
  const uint16_t *q;
  const void *pool;
  const float *scales;
  uint16_t *out;
  float *lse;
  float scale_log2;            // log2(e) / sqrt(D)
  int window, sinks;           // window: INT_MAX for all
};

__device__ __forceinline__ float4 decode4(uint32_t c) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)c));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(c >> 16)));
  const float2 a = __half22float2(*(const __half2 *)&lo), b = __half22float2(*(const __half2 *)&hi);
  return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ float4 bf16x4(uint2 u) {
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                     __uint_as_float(u.y & 0xffff0000u));
}
/* Channels 4 lane .. of a row of the pool. */
template <bool E4M3>
__device__ __forceinline__ float4 row4(const void *pool, size_t row, int lane, const float *scales) {
  if (!E4M3) return bf16x4(*((const uint2 *)((const uint16_t *)pool + row * D) + lane));
  const float4 x = decode4(*((const uint32_t *)((const uint8_t *)pool + row * D) + lane));
  const float s = scales[row / BLOCK];
  return make_float4(x.x * s, x.y * s, x.z * s, x.w * s);
}

constexpr int WARPS = 8;

/* A block per (sequence, layer, KV head), a warp per token in turn, a lane per four channels:
 * one pass with the running maximum and sum of each head. */
template <bool E4M3>
__global__ void __launch_bounds__(32 * WARPS) attend_cache_kernel(const __grid_constant__ AttendCacheParams p) {
  __shared__ float so[WARPS][GP][D], sm[WARPS][GP], sl[WARPS][GP];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int lh = p.L * p.Hkv, row = blockIdx.x;
  const int b = row / lh, l = row % lh / p.Hkv, h = row % p.Hkv;
  const int n = p.n_tokens[b], w0 = max(0, n - p.window), first = min(p.sinks, w0);
  const size_t q_row = ((size_t)b * p.L + l) * p.Hq + h * p.G;
  float4 q[GP], o[GP];
  float m[GP], z[GP];
#pragma unroll
  for (int i = 0; i < GP; ++i) {
    q[i] = i < p.G ? bf16x4(*((const uint2 *)(p.q + (q_row + i) * D) + lane)) : make_float4(0.f, 0.f, 0.f, 0.f);
    o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    m[i] = -INFINITY;
    z[i] = 0.f;
  }
  for (int j = warp; j < first + n - w0; j += WARPS) {
    const int tok = j < first ? j : j - first + w0, pg = tok / p.ps;
    const int phys = p.block_table[(size_t)b * p.P_max + pg];
    if ((unsigned)phys >= (unsigned)p.P_phys) continue;
    const size_t k_row = (((size_t)l * p.P_phys + phys) * p.Hkv + h) * 2 * p.ps + tok - pg * p.ps;
    const float4 k = row4<E4M3>(p.pool, k_row, lane, p.scales), v = row4<E4M3>(p.pool, k_row + p.ps, lane, p.scales);
#pragma unroll
    for (int i = 0; i < GP; ++i) {
      float s = (q[i].x * k.x + q[i].y * k.y) + (q[i].z * k.z + q[i].w * k.w);
#pragma unroll
      for (int e = 16; e; e >>= 1) s += __shfl_xor_sync(0xffffffffu, s, e);
      s *= p.scale_log2;
      const float top = fmaxf(m[i], s), base = top == -INFINITY ? 0.f : top;
      const float f = exp2f(m[i] - base), w = exp2f(s - base);
      m[i] = top;
      z[i] = z[i] * f + w;
      o[i] = make_float4(o[i].x * f + w * v.x, o[i].y * f + w * v.y, o[i].z * f + w * v.z, o[i].w * f + w * v.w);
    }
  }
#pragma unroll
  for (int i = 0; i < GP; ++i) {
    *(float4 *)&so[warp][i][4 * lane] = o[i];
    if (lane == 0) {
      sm[warp][i] = m[i];
      sl[warp][i] = z[i];
    }
  }
  __syncthreads();
  if (warp >= p.G) return;
  float top = -INFINITY, sum = 0.f;
  for (int y = 0; y < WARPS; ++y) top = fmaxf(top, sm[y][warp]);
  const float base = top == -INFINITY ? 0.f : top;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int y = 0; y < WARPS; ++y) {
    const float f = exp2f(sm[y][warp] - base);
    const float4 e = *(const float4 *)&so[y][warp][4 * lane];
    sum += f * sl[y][warp];
    acc = make_float4(acc.x + f * e.x, acc.y + f * e.y, acc.z + f * e.z, acc.w + f * e.w);
  }
  const float r = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;   // no token: zeros; NaN stays
  *(uint2 *)(p.out + (q_row + warp) * D + 4 * lane) =
      make_uint2(pack_bf16(acc.x * r, acc.y * r), pack_bf16(acc.z * r, acc.w * r));
  if (p.lse && lane == 0)
    p.lse[q_row + warp] = sum == 0.f ? -INFINITY : 0.69314718f * (base + log2f(sum));
}

}  // namespace

}  // namespace md

#define MD_API extern "C" __attribute__((visibility("default")))

MD_API md_status md_attend_cache(const md_attend_cache_args *args) {
  using namespace md;
  if (!args) return MD_ERR_INVALID_ARG;
  const md_attend_cache_args &a = *args;
  AttendCacheParams p;
  auto aligned = [](const void *x, size_t to) { return x && ((uintptr_t)x & (to - 1)) == 0; };
  const bool e4m3 = a.type == MD_TYPE_E4M3;
  if ((!e4m3 && a.type != MD_TYPE_BF16) || a.window < -1 || a.sinks < 0 || a.num_q_heads < 1 || !aligned(a.q_dev, 16) ||
      !aligned(a.pool_dev, 16) || (e4m3 && !aligned(a.scales_dev, 8)) || !aligned(a.block_table_dev, 4) ||
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
  p.scale_log2 = (float)(1.4426950408889634 / sqrt((double)D));
  p.window = a.window < 0 ? INT32_MAX : a.window;
  p.sinks = a.sinks;
  const dim3 grid((unsigned)(a.batch * a.num_layers * a.num_kv_heads));
  const auto kernel = e4m3 ? attend_cache_kernel<true> : attend_cache_kernel<false>;
  return launch_pdl(kernel, grid, 32 * WARPS, 0, (cudaStream_t)a.stream, p) == cudaSuccess ? MD_OK : MD_ERR_CUDA;
}
