/* A paged cache in eight bits: rows are quantised as they are written, and read back. */
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "md_internal.h"
#include "md_ptx.cuh"

namespace md {

namespace {

constexpr int BLOCK = MD_SCALE_TOKENS;

struct Cache8Params {
  void *rows[2];                         // k, v
  long long row[2], layer[2], head[2];   // their strides, in elements
  uint8_t *pool;
  float *scales;
  const int32_t *block_table;
  int L, Hkv, ps, P_phys, P_max, n_seqs;
  int first[MD_MAX_BATCH];               // position of a sequence's first row
  int row_start[MD_MAX_BATCH + 1];       // rows of the sequences before
  int block_start[MD_MAX_BATCH + 1];     // blocks of the sequences before
};

/* Four consecutive elements of a row, as they lie in memory and as fp32. */
template <class T>
struct Four {                            // bf16, f16
  uint2 u;
  __device__ __forceinline__ void load(const T *p) { u = *(const uint2 *)p; }
  __device__ __forceinline__ void store(T *p) const { *(uint2 *)p = u; }
};
template <>
struct Four<float> {
  float4 u;
  __device__ __forceinline__ void load(const float *p) { u = *(const float4 *)p; }
  __device__ __forceinline__ void store(float *p) const { *(float4 *)p = u; }
};
__device__ __forceinline__ float4 floats(const Four<__nv_bfloat16> &x) {
  return make_float4(__uint_as_float(x.u.x << 16), __uint_as_float(x.u.x & 0xffff0000u), __uint_as_float(x.u.y << 16),
                     __uint_as_float(x.u.y & 0xffff0000u));
}
__device__ __forceinline__ float4 floats(const Four<__half> &x) {
  const float2 a = __half22float2(*(const __half2 *)&x.u.x), b = __half22float2(*(const __half2 *)&x.u.y);
  return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ float4 floats(const Four<float> &x) { return x.u; }
__device__ __forceinline__ void round_to(Four<__nv_bfloat16> &y, float4 x) {
  y.u = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
}
__device__ __forceinline__ void round_to(Four<__half> &y, float4 x) {
  const __half2 a = __floats2half2_rn(x.x, x.y), b = __floats2half2_rn(x.z, x.w);
  y.u = make_uint2(*(const uint32_t *)&a, *(const uint32_t *)&b);
}
__device__ __forceinline__ void round_to(Four<float> &y, float4 x) { y.u = x; }

/* Four codes of four values; NaN stays NaN. */
__device__ __forceinline__ uint32_t encode4(float4 x) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x.y), "f"(x.x));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x.w), "f"(x.z));
  return (uint32_t)hi << 16 | lo;
}
__device__ __forceinline__ float4 decode4(uint32_t c) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)c));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(c >> 16)));
  const float2 a = __half22float2(*(const __half2 *)&lo), b = __half22float2(*(const __half2 *)&hi);
  return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ float4 times(float4 x, float s) { return make_float4(x.x * s, x.y * s, x.z * s, x.w * s); }

/* A block's part of a call: a warp per (block of 16 tokens, layer, KV head, K or V), a lane per
 * four channels of its rows. */
struct Unit {
  int which, layer, head;      // K: 0, V: 1
  int lo, hi;                  // slots of the block that the call is about
  long long row;               // the row of slot 0 (before the first one, if the block begins earlier)
  uint8_t *codes;              // of slot 0
  float *scale;                // null: not in the pool
};
__device__ __forceinline__ Unit unit_of(const Cache8Params &p, long long u) {
  Unit r;
  r.which = (int)(u & 1);
  u >>= 1;
  r.head = (int)(u % p.Hkv);
  u /= p.Hkv;
  const int blocks = p.block_start[p.n_seqs];
  r.layer = (int)(u / blocks);
  const int at = (int)(u - (long long)r.layer * blocks);
  int b = 0, hi = p.n_seqs;              // the sequence: block_start[b] <= at < block_start[b + 1]
  while (hi - b > 1) {
    const int mid = (b + hi) >> 1;
    if (p.block_start[mid] <= at) b = mid;
    else hi = mid;
  }
  const int first = p.first[b], count = p.row_start[b + 1] - p.row_start[b];
  const int block = first / BLOCK + at - p.block_start[b], tok = block * BLOCK;
  r.lo = max(first - tok, 0);
  r.hi = min(first + count - tok, BLOCK);
  r.row = (long long)p.row_start[b] + tok - first;
  const int pg = tok / p.ps, part = (tok - pg * p.ps) / BLOCK;
  const int phys = p.block_table[(size_t)b * p.P_max + pg];
  const bool in = (unsigned)phys < (unsigned)p.P_phys;
  const size_t rows = ((((size_t)r.layer * p.P_phys + (in ? phys : 0)) * p.Hkv + r.head) * 2 + r.which) * p.ps + part * BLOCK;
  r.codes = p.pool + rows * D;
  r.scale = in ? p.scales + rows / BLOCK : nullptr;
  return r;
}

/* The scale is a power of two: x / s and the codes of a block that moves to a larger scale
 * are then exact (but for subnormal codes), and a float code has the same relative precision in
 * every binade, so that a scale of max / 448 would gain nothing but part of a binade at the
 * small end. */
template <class T>
__global__ void __launch_bounds__(256) write_cache8_kernel(const __grid_constant__ Cache8Params p) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long units = (long long)p.block_start[p.n_seqs] * p.L * p.Hkv * 2;
  for (long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += (long long)gridDim.x * 8) {
    const Unit t = unit_of(p, u);
    if (!t.scale) continue;
    const T *src = (const T *)p.rows[t.which] + t.row * p.row[t.which] + t.layer * p.layer[t.which] +
                   t.head * p.head[t.which] + 4 * lane;
    const float before = t.lo > 0 ? *t.scale : 0.f;
    Four<T> x[BLOCK];
#pragma unroll
    for (int r = 0; r < BLOCK; ++r)
      if (r >= t.lo && r < t.hi) x[r].load(src + r * p.row[t.which]);
    float most = 0.f;                    // of the finite values
#pragma unroll
    for (int r = 0; r < BLOCK; ++r)
      if (r >= t.lo && r < t.hi) {
        const float4 f = floats(x[r]);
        auto size = [](float v) { return fabsf(v) < INFINITY ? fabsf(v) : 0.f; };
        most = fmaxf(fmaxf(most, fmaxf(size(f.x), size(f.y))), fmaxf(size(f.z), size(f.w)));
      }
    /* 448 is 1.75 x 2^8: fractions above 1.75 carry into the next exponent */
    const uint32_t bits = __reduce_max_sync(0xffffffffu, __float_as_uint(most)) + 0x1fffffu;
    const float least = __uint_as_float(max((int)(bits >> 23) - 8, 1) << 23);
    const float scale = fmaxf(before, least), inv = 1.f / scale;
    uint32_t *dst = (uint32_t *)t.codes + lane;
    if (t.lo > 0 && scale > before) {
      const float ratio = before * inv;
#pragma unroll
      for (int r = 0; r < BLOCK; ++r)
        if (r < t.lo) dst[r * (D / 4)] = encode4(times(decode4(dst[r * (D / 4)]), ratio));
    }
#pragma unroll
    for (int r = 0; r < BLOCK; ++r)
      if (r >= t.lo && r < t.hi) {
        const float4 f = floats(x[r]);
        auto code = [&](float v) { return fmaf(v, 0.f, v * inv); };   // infinities become NaN
        dst[r * (D / 4)] = encode4(make_float4(code(f.x), code(f.y), code(f.z), code(f.w)));
      }
    if (lane == 0 && scale != before) *t.scale = scale;
  }
}

template <class T>
__global__ void __launch_bounds__(256) read_cache8_kernel(const __grid_constant__ Cache8Params p) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long units = (long long)p.block_start[p.n_seqs] * p.L * p.Hkv * 2;
  for (long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += (long long)gridDim.x * 8) {
    const Unit t = unit_of(p, u);
    T *dst = (T *)p.rows[t.which] + t.row * p.row[t.which] + t.layer * p.layer[t.which] + t.head * p.head[t.which] + 4 * lane;
    const uint32_t *src = (const uint32_t *)t.codes + lane;
    uint32_t c[BLOCK];
#pragma unroll
    for (int r = 0; r < BLOCK; ++r) c[r] = t.scale && r >= t.lo && r < t.hi ? src[r * (D / 4)] : 0x7f7f7f7fu;
    const float scale = t.scale ? *t.scale : 1.f;
#pragma unroll
    for (int r = 0; r < BLOCK; ++r)
      if (r >= t.lo && r < t.hi) {
        Four<T> y;
        round_to(y, times(decode4(c[r]), scale));
        y.store(dst + r * p.row[t.which]);
      }
  }
}

bool aligned(const void *p, size_t a) { return p && ((uintptr_t)p & (a - 1)) == 0; }

/* The checks of both calls, and their launches' parameters. */
md_status cache8_params(const md_cache8_args *args, Cache8Params &p) {
  if (!args || !args->first_host || !args->count_host || args->batch < 1 || args->batch > MD_MAX_BATCH)
    return MD_ERR_INVALID_ARG;
  const md_cache8_args &a = *args;
  if (a.type < MD_TYPE_BF16 || a.type > MD_TYPE_F32) return MD_ERR_INVALID_ARG;
  const long long limit = (long long)MD_MAX_CHUNKS * MD_MAX_CHUNK_TOKENS;
  int32_t n[MD_MAX_BATCH];
  for (int b = 0; b < a.batch; ++b) {
    if (a.first_host[b] < 0 || a.count_host[b] < 0 || (long long)a.first_host[b] + a.count_host[b] > limit)
      return MD_ERR_INVALID_ARG;
    n[b] = a.first_host[b] + a.count_host[b];
  }
  PageSet s;
  if (!a.block_table_dev ||
      !page_set(s, a.block_table_dev, n, a.batch, a.num_layers, 0, a.num_kv_heads, a.page_size, a.max_pages_per_seq,
                a.num_phys_pages))
    return MD_ERR_INVALID_ARG;
  const size_t base = a.type == MD_TYPE_F32 ? 16 : 8;
  if (!aligned(a.pool_dev, 16) || !aligned(a.scales_dev, 8) || !aligned(a.block_table_dev, 4)) return MD_ERR_INVALID_ARG;
  if ((a.k_row | a.k_layer | a.k_head | a.v_row | a.v_layer | a.v_head) & 3) return MD_ERR_INVALID_ARG;
  p.rows[0] = a.k;
  p.rows[1] = a.v;
  p.row[0] = a.k_row;
  p.row[1] = a.v_row;
  p.layer[0] = a.k_layer;
  p.layer[1] = a.v_layer;
  p.head[0] = a.k_head;
  p.head[1] = a.v_head;
  p.pool = (uint8_t *)a.pool_dev;
  p.scales = a.scales_dev;
  p.block_table = a.block_table_dev;
  p.L = a.num_layers;
  p.Hkv = a.num_kv_heads;
  p.ps = a.page_size;
  p.P_phys = a.num_phys_pages;
  p.P_max = a.max_pages_per_seq;
  p.n_seqs = a.batch;
  p.row_start[0] = p.block_start[0] = 0;
  for (int b = 0; b < a.batch; ++b) {
    p.first[b] = a.first_host[b];
    p.row_start[b + 1] = p.row_start[b] + a.count_host[b];       // 256 sequences of 2^18 tokens at most
    p.block_start[b + 1] = p.block_start[b] + (a.count_host[b] ? (n[b] - 1) / BLOCK - p.first[b] / BLOCK + 1 : 0);
  }
  if (p.row_start[a.batch] > 0 && (!aligned(a.k, base) || !aligned(a.v, base))) return MD_ERR_INVALID_ARG;
  return MD_OK;
}

template <class F>
md_status launch(const Cache8Params &p, int type, void *stream, F kernels) {
  const long long units = (long long)p.block_start[p.n_seqs] * p.L * p.Hkv * 2, blocks = (units + 7) / 8;
  if (units == 0) return MD_OK;
  const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20));
  return launch_pdl(kernels(type), grid, 256, 0, (cudaStream_t)stream, p) == cudaSuccess ? MD_OK : MD_ERR_CUDA;
}

}  // namespace

}  // namespace md

#define MD_API extern "C" __attribute__((visibility("default")))

MD_API md_status md_write_cache8(const md_cache8_args *args) {
  using namespace md;
  Cache8Params p;
  const md_status st = cache8_params(args, p);
  if (st != MD_OK) return st;
  return launch(p, args->type, args->stream, [](int type) {
    return type == MD_TYPE_BF16  ? write_cache8_kernel<__nv_bfloat16>
           : type == MD_TYPE_F16 ? write_cache8_kernel<__half>
                                 : write_cache8_kernel<float>;
  });
}

MD_API md_status md_read_cache8(const md_cache8_args *args) {
  using namespace md;
  Cache8Params p;
  const md_status st = cache8_params(args, p);
  if (st != MD_OK) return st;
  return launch(p, args->type, args->stream, [](int type) {
    return type == MD_TYPE_BF16  ? read_cache8_kernel<__nv_bfloat16>
           : type == MD_TYPE_F16 ? read_cache8_kernel<__half>
                                 : read_cache8_kernel<float>;
  });
}
