/* A paged cache in eight bits: rows are quantised as they are written, and read back. */
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "md_internal.h"
#include "md_ptx.cuh"

namespace md {

namespace {

constexpr int BLOCK = MD_SCALE_TOKENS;

/* N: sequences that there is room for.  Few sequences take small parameters: a call that writes one
 * token takes 3.1 us of the host instead of 3.6. */
constexpr int FEW = 16;
template <int N>
struct Cache8Params {
  void *rows[2];                         // k, v
  long long row[2], layer[2], head[2];   // their strides, in elements
  uint8_t *pool;
  float *scales;
  const int32_t *block_table;
  int L, Hkv, ps, P_phys, P_max, n_seqs;
  int first[N];                          // position of a sequence's first row
  int row_start[N + 1];                  // rows of the sequences before
  int block_start[N + 1];                // blocks of the sequences before
};

/* W consecutive elements of a row, as they lie in memory. */
template <class T, int W>
struct Piece {
  static constexpr int WORDS = W * (int)sizeof(T) / 4;
  uint32_t w[WORDS];
  __device__ __forceinline__ void load(const T *p) {
    if constexpr (WORDS == 2) {
      const uint2 u = *(const uint2 *)p;
      w[0] = u.x, w[1] = u.y;
    } else {
      const uint4 u = *(const uint4 *)p;
      w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
    }
  }
  __device__ __forceinline__ void store(T *p) const {
    if constexpr (WORDS == 2) *(uint2 *)p = make_uint2(w[0], w[1]);
    else *(uint4 *)p = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

/* Per type: a word's elements as fp32, and back; the larger sizes of two words' elements, as
 * integers, which order like them with what is not finite on top. */
template <class T>
struct Type;
template <>
struct Type<__nv_bfloat16> {
  static constexpr int PER_WORD = 2;
  static constexpr uint32_t SIGNS = 0x80008000u;
  static __device__ __forceinline__ void floats(uint32_t w, float *f) {
    f[0] = __uint_as_float(w << 16);
    f[1] = __uint_as_float(w & 0xffff0000u);
  }
  static __device__ __forceinline__ uint32_t word(const float *f) { return pack_bf16(f[0], f[1]); }
  static __device__ __forceinline__ float size(uint32_t bits) { return __uint_as_float(bits << 16); }
};
template <>
struct Type<__half> {
  static constexpr int PER_WORD = 2;
  static constexpr uint32_t SIGNS = 0x80008000u;
  static __device__ __forceinline__ void floats(uint32_t w, float *f) {
    const float2 x = __half22float2(*(const __half2 *)&w);
    f[0] = x.x;
    f[1] = x.y;
  }
  static __device__ __forceinline__ uint32_t word(const float *f) {
    const __half2 x = __floats2half2_rn(f[0], f[1]);
    return *(const uint32_t *)&x;
  }
  static __device__ __forceinline__ float size(uint32_t bits) {
    float f[2];
    floats(bits, f);
    return f[0];
  }
};
template <>
struct Type<float> {
  static constexpr int PER_WORD = 1;
  static constexpr uint32_t SIGNS = 0x80000000u;
  static __device__ __forceinline__ void floats(uint32_t w, float *f) { f[0] = __uint_as_float(w); }
  static __device__ __forceinline__ uint32_t word(const float *f) { return __float_as_uint(f[0]); }
  static __device__ __forceinline__ float size(uint32_t bits) { return __uint_as_float(bits); }
};
template <class T>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  if constexpr (Type<T>::PER_WORD == 1) return max(a, b);
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

/* Codes of four values; NaN stays NaN. */
__device__ __forceinline__ uint32_t encode4(const float *x) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x[1]), "f"(x[0]));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x[3]), "f"(x[2]));
  return (uint32_t)hi << 16 | lo;
}
__device__ __forceinline__ void decode4(uint32_t c, float s, float *x) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)c));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(c >> 16)));
  const float2 a = __half22float2(*(const __half2 *)&lo), b = __half22float2(*(const __half2 *)&hi);
  x[0] = a.x * s, x[1] = a.y * s, x[2] = b.x * s, x[3] = b.y * s;
}
/* W codes of a row. */
template <int W>
struct Codes {
  uint32_t c[W / 4];
  __device__ __forceinline__ void load(const uint8_t *p) {
    if constexpr (W == 4) {
      c[0] = *(const uint32_t *)p;
    } else {
      const uint2 u = *(const uint2 *)p;
      c[0] = u.x, c[1] = u.y;
    }
  }
  __device__ __forceinline__ void store(uint8_t *p) const {
    if constexpr (W == 4) *(uint32_t *)p = c[0];
    else *(uint2 *)p = make_uint2(c[0], c[1]);
  }
};

/* A block's part of a call: a warp per (layer, block of 16 tokens, KV head, K or V), a lane per W
 * channels of every (32 W / 128)th of its rows. */
struct Unit {
  int which;                   // K: 0, V: 1
  int lo, hi;                  // slots of the block that the call is about
  long long at;                // of slot 0 in the rows (before them, if the block begins earlier)
  uint8_t *codes;              // of slot 0
  float *scale;                // null: not in the pool
};
template <int N>
__device__ __forceinline__ bool unit_of(const Cache8Params<N> &p, Unit &r) {
  const unsigned v = blockIdx.x * 8 + (threadIdx.x >> 5), per = 2 * p.Hkv;
  const int at = (int)(v / per), hw = (int)(v - at * per), layer = blockIdx.y, head = hw >> 1;
  if (at >= p.block_start[p.n_seqs]) return false;
  int b = 0;                             // the sequence: block_start[b] <= at < block_start[b + 1]
  for (int hi = p.n_seqs; hi - b > 1;) {
    const int mid = (b + hi) >> 1;
    if (p.block_start[mid] <= at) b = mid;
    else hi = mid;
  }
  r.which = hw & 1;
  const int first = p.first[b], count = p.row_start[b + 1] - p.row_start[b];
  const int tok = (first / BLOCK + at - p.block_start[b]) * BLOCK;
  r.lo = max(first - tok, 0);
  r.hi = min(first + count - tok, BLOCK);
  r.at = ((long long)p.row_start[b] + tok - first) * p.row[r.which] + layer * p.layer[r.which] + head * p.head[r.which];
  const int pg = p.ps == 16 ? tok >> 4 : tok >> 5, part = (tok & (p.ps - 1)) / BLOCK;
  const int phys = p.block_table[(size_t)b * p.P_max + pg];
  const bool in = (unsigned)phys < (unsigned)p.P_phys;
  const size_t rows = ((((size_t)layer * p.P_phys + (in ? phys : 0)) * p.Hkv + head) * 2 + r.which) * p.ps + part * BLOCK;
  r.codes = p.pool + rows * D;
  r.scale = in ? p.scales + rows / BLOCK : nullptr;
  return true;
}

/* The scale is a power of two: x / s and the codes of a block that moves to a larger scale
 * are then exact (but for subnormal codes), and a float code has the same relative precision in
 * every binade, so that a scale of max / 448 would gain nothing but part of a binade at the
 * small end. */
template <class T, int W, int SEQS>
__global__ void __launch_bounds__(256) write_cache8_kernel(const __grid_constant__ Cache8Params<SEQS> p) {
  using X = Type<T>;
  constexpr int R = 32 * W / D, N = BLOCK / R;       // rows of the warp at once, rows of a lane
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, row0 = lane / (D / W), d = lane % (D / W) * W;
  Unit t;
  if (!unit_of(p, t) || !t.scale) return;
  const T *src = (const T *)p.rows[t.which] + t.at + d;
  const float before = t.lo > 0 ? *t.scale : 0.f;
  Piece<T, W> x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = R * i + row0;
    if (r >= t.lo && r < t.hi) {
      x[i].load(src + r * p.row[t.which]);
    } else {
#pragma unroll
      for (int k = 0; k < Piece<T, W>::WORDS; ++k) x[i].w[k] = 0;
    }
  }
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int k = 0; k < Piece<T, W>::WORDS; ++k) most = larger<T>(most, x[i].w[k] & ~X::SIGNS);
  if (X::PER_WORD == 2) most = max(most >> 16, most & 0xffffu);
  float size = X::size(__reduce_max_sync(0xffffffffu, most));
  const bool odd = !(size < INFINITY);               // something is not finite: it is left out
  if (odd) {
    size = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int k = 0; k < Piece<T, W>::WORDS; ++k) {
        float f[2] = {0.f, 0.f};
        X::floats(x[i].w[k], f);
        size = fmaxf(size, fmaxf(fabsf(f[0]) < INFINITY ? fabsf(f[0]) : 0.f, fabsf(f[1]) < INFINITY ? fabsf(f[1]) : 0.f));
      }
    size = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(size)));
  }
  /* 448 is 1.75 x 2^8: fractions above 1.75 carry into the next exponent */
  const float least = __uint_as_float(max((int)(__float_as_uint(size) + 0x1fffffu >> 23) - 8, 1) << 23);
  const float scale = fmaxf(before, least), inv = 1.f / scale;
  uint8_t *dst = t.codes + d;
  if (t.lo > 0 && scale > before) {
    const float ratio = before * inv;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = R * i + row0;
      if (r >= t.lo) continue;
      Codes<W> c;
      c.load(dst + r * D);
#pragma unroll
      for (int k = 0; k < W / 4; ++k) {
        float f[4];
        decode4(c.c[k], ratio, f);
        c.c[k] = encode4(f);
      }
      c.store(dst + r * D);
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = R * i + row0;
    if (r < t.lo || r >= t.hi) continue;
    float f[W];
#pragma unroll
    for (int k = 0; k < Piece<T, W>::WORDS; ++k) X::floats(x[i].w[k], f + k * X::PER_WORD);
    if (odd) {
#pragma unroll
      for (int k = 0; k < W; ++k) f[k] = fmaf(f[k], 0.f, f[k]);      // infinities become NaN
    }
    Codes<W> c;
#pragma unroll
    for (int k = 0; k < W; ++k) f[k] *= inv;
#pragma unroll
    for (int k = 0; k < W / 4; ++k) c.c[k] = encode4(f + 4 * k);
    c.store(dst + r * D);
  }
  if (lane == 0 && scale != before) *t.scale = scale;
}

template <class T, int W, int SEQS>
__global__ void __launch_bounds__(256) read_cache8_kernel(const __grid_constant__ Cache8Params<SEQS> p) {
  using X = Type<T>;
  constexpr int R = 32 * W / D, N = BLOCK / R;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, row0 = lane / (D / W), d = lane % (D / W) * W;
  Unit t;
  if (!unit_of(p, t)) return;
  T *dst = (T *)p.rows[t.which] + t.at + d;
  Codes<W> c[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = R * i + row0;
    if (t.scale && r >= t.lo && r < t.hi) {
      c[i].load(t.codes + r * D + d);
    } else {
#pragma unroll
      for (int k = 0; k < W / 4; ++k) c[i].c[k] = 0x7f7f7f7fu;
    }
  }
  const float scale = t.scale ? *t.scale : 1.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = R * i + row0;
    if (r < t.lo || r >= t.hi) continue;
    float f[W];
#pragma unroll
    for (int k = 0; k < W / 4; ++k) decode4(c[i].c[k], scale, f + 4 * k);
    Piece<T, W> y;
#pragma unroll
    for (int k = 0; k < Piece<T, W>::WORDS; ++k) y.w[k] = X::word(f + k * X::PER_WORD);
    y.store(dst + r * p.row[t.which]);
  }
}

bool aligned(const void *p, size_t a) { return p && ((uintptr_t)p & (a - 1)) == 0; }

/* The checks of both calls, and their launches' parameters. */
template <int N>
md_status cache8_params(const md_cache8_args &a, Cache8Params<N> &p) {
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
  if (!aligned(a.pool_dev, 16) || !aligned(a.scales_dev, 4) || !aligned(a.block_table_dev, 4)) return MD_ERR_INVALID_ARG;
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

/* Rows of two-byte elements that are aligned to 16 bytes go 16 bytes at a time. */
template <int N>
bool wide(const Cache8Params<N> &p) {
  for (int i = 0; i < 2; ++i)
    if (!aligned(p.rows[i], 16) || ((p.row[i] | p.layer[i] | p.head[i]) & 7)) return false;
  return true;
}

template <int N, bool WRITE>
md_status cache8(const md_cache8_args &a) {
  Cache8Params<N> p;
  const md_status st = cache8_params(a, p);
  if (st != MD_OK) return st;
  const long long units = (long long)p.block_start[p.n_seqs] * p.Hkv * 2;
  if (units == 0) return MD_OK;
  if (units >= 1LL << 31) return MD_ERR_INVALID_ARG;
  const dim3 grid((unsigned)((units + 7) / 8), p.L);
  auto launch = [&](auto write, auto read) {
    return launch_pdl(WRITE ? write : read, grid, 256, 0, (cudaStream_t)a.stream, p) == cudaSuccess ? MD_OK : MD_ERR_CUDA;
  };
  if (a.type == MD_TYPE_F32) return launch(write_cache8_kernel<float, 4, N>, read_cache8_kernel<float, 4, N>);
  const bool w = wide(p);
  if (a.type == MD_TYPE_BF16)
    return w ? launch(write_cache8_kernel<__nv_bfloat16, 8, N>, read_cache8_kernel<__nv_bfloat16, 8, N>)
             : launch(write_cache8_kernel<__nv_bfloat16, 4, N>, read_cache8_kernel<__nv_bfloat16, 4, N>);
  return w ? launch(write_cache8_kernel<__half, 8, N>, read_cache8_kernel<__half, 8, N>)
           : launch(write_cache8_kernel<__half, 4, N>, read_cache8_kernel<__half, 4, N>);
}

template <bool WRITE>
md_status cache8(const md_cache8_args *a) {
  if (!a || !a->first_host || !a->count_host || a->batch < 1 || a->batch > MD_MAX_BATCH) return MD_ERR_INVALID_ARG;
  return a->batch <= FEW ? cache8<FEW, WRITE>(*a) : cache8<MD_MAX_BATCH, WRITE>(*a);
}

}  // namespace

}  // namespace md

#define MD_API extern "C" __attribute__((visibility("default")))

MD_API md_status md_write_cache8(const md_cache8_args *args) { return md::cache8<true>(args); }

MD_API md_status md_read_cache8(const md_cache8_args *args) { return md::cache8<false>(args); }
