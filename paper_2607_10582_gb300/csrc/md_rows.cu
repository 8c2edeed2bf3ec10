/* A layer's rows on their way into the cache: head norms, rotation by position,
 * and the layouts of md_decode_* and md_append_tokens, in one pass. */
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <string.h>

#include "md_internal.h"
#include "md_ptx.cuh"

namespace md {

namespace {

struct RowsParams {
  md_norm_rope_args a;
  int parts, rows_per_part;   // a token's rows are split over `parts` half-warps
  uint8_t axis[D / 2];
};

/* 4 consecutive elements, as they are and as fp32 */
template <class T>
struct Raw {
  typedef uint2 type;
};
template <>
struct Raw<float> {
  typedef float4 type;
};
__device__ __forceinline__ void widen(const uint2 &u, float (&x)[4], __nv_bfloat16) {
  x[0] = __uint_as_float(u.x << 16);
  x[1] = __uint_as_float(u.x & 0xffff0000u);
  x[2] = __uint_as_float(u.y << 16);
  x[3] = __uint_as_float(u.y & 0xffff0000u);
}
__device__ __forceinline__ void widen(const uint2 &u, float (&x)[4], __half) {
  const float2 a = __half22float2(*(const __half2 *)&u.x), b = __half22float2(*(const __half2 *)&u.y);
  x[0] = a.x;
  x[1] = a.y;
  x[2] = b.x;
  x[3] = b.y;
}
__device__ __forceinline__ void widen(const float4 &u, float (&x)[4], float) {
  x[0] = u.x;
  x[1] = u.y;
  x[2] = u.z;
  x[3] = u.w;
}
__device__ __forceinline__ void store4(uint16_t *p, const float (&x)[4]) {
  *(uint2 *)p = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
}

/* A half-warp per token, or per part of a token's rows: what the rows share
 * (table entries, weights) is loaded once.  A row is eight elements per lane, two
 * groups of four, chosen so that a lane holds both channels of its four pairs:
 * 4j .. and R/2 + 4j .. for the pairs (i, i + R/2), 8j .. 8j + 7 for (2i, 2i + 1);
 * lanes past the rotated channels hold the rest.  Four rows are in flight. */
template <class T>
__global__ void __launch_bounds__(256) norm_rope_kernel(const __grid_constant__ RowsParams p) {
  typedef typename Raw<T>::type raw;
  constexpr int FLIGHT = 4;
  pdl_wait();
  pdl_trigger();
  const md_norm_rope_args &a = p.a;
  const int j = threadIdx.x & 15;
  const long long unit = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (unit >= (long long)a.n_tokens * p.parts) return;   // whole half-warps; the shuffles stay inside them
  const unsigned half = threadIdx.x & 16 ? 0xffff0000u : 0xffffu;
  const long long tok = unit / p.parts;
  const int first = (int)(unit - tok * p.parts) * p.rows_per_part;   // of the token's q, k and v rows, in this order
  const int R = a.rotary_dim;
  const bool rot = 8 * j < R;
  const int e0 = a.interleaved || !rot ? 8 * j : 4 * j, e1 = a.interleaved || !rot ? e0 + 4 : R / 2 + 4 * j;
  float c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f};
  if (rot) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pos = a.positions[(size_t)p.axis[4 * j + i] * a.n_tokens + tok];
      float2 cs = make_float2(NAN, NAN);
      if (pos >= 0 && pos < a.table_len) cs = ((const float2 *)a.table)[(size_t)pos * (R / 2) + 4 * j + i];
      c[i] = cs.x;
      s[i] = cs.y;
    }
  }
  /* rows lo .. hi - 1 of one of q, k, v */
  auto rows = [&](const void *in, int64_t in_token, int64_t in_head, void *out, int64_t out_token, int64_t out_head,
                  const float *w, bool value, int lo, int hi) {
    const T *src = (const T *)in + tok * in_token;
    uint16_t *dst = (uint16_t *)out + tok * out_token;
    float wx[4], wy[4];
    if (w) {
      widen(*(const float4 *)(w + e0), wx, 0.f);
      widen(*(const float4 *)(w + e1), wy, 0.f);
    }
    for (int h0 = lo; h0 < hi; h0 += FLIGHT) {
      raw u[FLIGHT], v[FLIGHT];
#pragma unroll
      for (int r = 0; r < FLIGHT; ++r) {
        const T *x = src + min(h0 + r, hi - 1) * in_head;
        u[r] = *(const raw *)(x + e0);
        v[r] = *(const raw *)(x + e1);
      }
#pragma unroll
      for (int r = 0; r < FLIGHT; ++r) {
        if (h0 + r >= hi) break;
        float x[4], y[4];
        widen(u[r], x, T());
        widen(v[r], y, T());
        if (w) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) sum += x[i] * x[i] + y[i] * y[i];
#pragma unroll
          for (int o = 8; o; o >>= 1) sum += __shfl_xor_sync(half, sum, o);
          const float f = rsqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[i] *= f * wx[i];
            y[i] *= f * wy[i];
          }
        }
        if (rot && !value) {
          float n[4], m[4];
          if (a.interleaved) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              n[2 * i] = x[2 * i] * c[i] - x[2 * i + 1] * s[i];
              n[2 * i + 1] = x[2 * i + 1] * c[i] + x[2 * i] * s[i];
              m[2 * i] = y[2 * i] * c[i + 2] - y[2 * i + 1] * s[i + 2];
              m[2 * i + 1] = y[2 * i + 1] * c[i + 2] + y[2 * i] * s[i + 2];
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              n[i] = x[i] * c[i] - y[i] * s[i];
              m[i] = y[i] * c[i] + x[i] * s[i];
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[i] = n[i];
            y[i] = m[i];
          }
        }
        uint16_t *d = dst + (h0 + r) * out_head;
        store4(d + e0, x);
        store4(d + e1, y);
      }
    }
  };
  const int last = first + p.rows_per_part, Hq = a.num_q_heads, Hkv = a.num_kv_heads;
  auto clip = [&](int n, int at) { return max(0, min(n, at)); };
  rows(a.q, a.q_token, a.q_head, a.q_out, a.q_out_token, a.q_out_head, a.q_weight, false, clip(Hq, first), clip(Hq, last));
  rows(a.k, a.k_token, a.k_head, a.k_out, a.k_out_token, a.k_out_head, a.k_weight, false, clip(Hkv, first - Hq),
       clip(Hkv, last - Hq));
  if (a.v)
    rows(a.v, a.v_token, a.v_head, a.v_out, a.v_out_token, a.v_out_head, nullptr, true, clip(Hkv, first - Hq - Hkv),
         clip(Hkv, last - Hq - Hkv));
}

struct TableParams {
  float2 *table;
  int pairs, len;
  double scale;
  double freq[D / 2];
};

__global__ void __launch_bounds__(256) rope_table_kernel(const __grid_constant__ TableParams p) {
  pdl_wait();
  pdl_trigger();
  const long long n = (long long)p.len * p.pairs;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    double s, c;
    sincos((double)(i / p.pairs) * p.freq[i % p.pairs], &s, &c);
    p.table[i] = make_float2((float)(p.scale * c), (float)(p.scale * s));
  }
}

constexpr int UNITS = 152 * 128;

bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
bool rows_ok(const void *p, int64_t token, int64_t head, size_t align) {
  return p && aligned(p, align) && token % 4 == 0 && head % 4 == 0;
}

}  // namespace

}  // namespace md

#define MD_API extern "C" __attribute__((visibility("default")))

MD_API md_status md_rope_table(const double *inv_freq, int rotary_dim, int table_len, double scale, float *table,
                               void *stream) {
  using namespace md;
  if (!inv_freq || !table || !aligned(table, 16) || rotary_dim < 8 || rotary_dim > D || rotary_dim % 8 ||
      table_len < 1)
    return MD_ERR_INVALID_ARG;
  TableParams p;
  p.table = (float2 *)table;
  p.pairs = rotary_dim / 2;
  p.len = table_len;
  p.scale = scale;
  memcpy(p.freq, inv_freq, p.pairs * sizeof(double));
  const long long blocks = ((long long)table_len * p.pairs + 255) / 256;
  const cudaError_t e =
      launch_pdl(rope_table_kernel, (int)(blocks < 4096 ? blocks : 4096), 256, 0, (cudaStream_t)stream, p);
  return e == cudaSuccess ? MD_OK : MD_ERR_CUDA;
}

MD_API md_status md_norm_rope(const md_norm_rope_args *args) {
  using namespace md;
  if (!args) return MD_ERR_INVALID_ARG;
  RowsParams p;
  p.a = *args;
  md_norm_rope_args &a = p.a;
  if (a.n_tokens < 0 || a.num_q_heads < 0 || a.num_kv_heads < 0 || a.num_q_heads > 65535 || a.num_kv_heads > 65535 ||
      a.type < MD_TYPE_BF16 || a.type > MD_TYPE_F32 || a.rotary_dim < 0 || a.rotary_dim > D || a.rotary_dim % 8 ||
      !(a.eps >= 0.f))
    return MD_ERR_INVALID_ARG;
  const size_t in = a.type == MD_TYPE_F32 ? 16 : 8;
  if (a.num_q_heads > 0 && (!rows_ok(a.q, a.q_token, a.q_head, in) || !rows_ok(a.q_out, a.q_out_token, a.q_out_head, 8)))
    return MD_ERR_INVALID_ARG;
  if (a.num_kv_heads > 0) {
    if (!rows_ok(a.k, a.k_token, a.k_head, in) || !rows_ok(a.k_out, a.k_out_token, a.k_out_head, 8))
      return MD_ERR_INVALID_ARG;
    if (a.v && (!rows_ok(a.v, a.v_token, a.v_head, in) || !rows_ok(a.v_out, a.v_out_token, a.v_out_head, 8)))
      return MD_ERR_INVALID_ARG;
  }
  if (!aligned(a.q_weight, 16) || !aligned(a.k_weight, 16)) return MD_ERR_INVALID_ARG;
  memset(p.axis, 0, sizeof(p.axis));
  if (a.rotary_dim > 0) {
    if (!a.table || !aligned(a.table, 16) || !a.positions || a.num_axes < 1 || a.num_axes > MD_MAX_AXES || a.table_len < 1)
      return MD_ERR_INVALID_ARG;
    for (int i = 0; a.axis_host && i < a.rotary_dim / 2; ++i) {
      if (a.axis_host[i] >= a.num_axes) return MD_ERR_INVALID_ARG;
      p.axis[i] = a.axis_host[i];
    }
  }
  const int rows = a.num_q_heads + a.num_kv_heads * (a.v ? 2 : 1);
  if (a.n_tokens == 0 || rows == 0) return MD_OK;
  /* as many parts as keep about UNITS half-warps busy */
  p.parts = (int)(UNITS / a.n_tokens < 1 ? 1 : UNITS / a.n_tokens > rows ? rows : UNITS / a.n_tokens);
  p.rows_per_part = (rows + p.parts - 1) / p.parts;
  p.parts = (rows + p.rows_per_part - 1) / p.rows_per_part;
  const long long blocks = ((long long)a.n_tokens * p.parts + 15) / 16;
  if (blocks >= (1LL << 31)) return MD_ERR_INVALID_ARG;
  const cudaStream_t s = (cudaStream_t)a.stream;
  cudaError_t e;
  if (a.type == MD_TYPE_BF16)
    e = launch_pdl(norm_rope_kernel<__nv_bfloat16>, (int)blocks, 256, 0, s, p);
  else if (a.type == MD_TYPE_F16)
    e = launch_pdl(norm_rope_kernel<__half>, (int)blocks, 256, 0, s, p);
  else
    e = launch_pdl(norm_rope_kernel<float>, (int)blocks, 256, 0, s, p);
  return e == cudaSuccess ? MD_OK : MD_ERR_CUDA;
}
