/* A layer's rows on their way into the cache: head norms, rotation by position,
 * and the layouts of md_decode_* and md_append_tokens, in one pass. */
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <string.h>

#include <algorithm>

#include "md_internal.h"
#include "md_ptx.cuh"

namespace md {

namespace {

/* The rows of q, k and v: element (token, head, d) is at token * token_stride +
 * head * head_stride + d. */
struct Rows {
  const void *in;
  uint16_t *out;
  const float *weight;        // null: no norm
  long long in_token, in_head, out_token, out_head;
  int heads, rotate;
};
struct RowsParams {
  Rows set[3];
  const float2 *table;
  const int32_t *positions;
  long long n_tokens;
  int table_len, rotary_dim;
  float eps;
  int split_log;              // a token's rows are split over 2^split_log units (4 at least)
  unsigned long long axes[2]; // the axis of pair q: 2 bits at 2 (q % 32) of word q / 32
};

/* ---- pairs of fp32 in one 64-bit register, two results per instruction ---- */
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 parts(f32x2 x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

/* Two consecutive elements as fp32. */
__device__ __forceinline__ f32x2 load2(const __nv_bfloat16 *p) {
  const uint32_t u = *(const uint32_t *)p;
  return pair(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
__device__ __forceinline__ f32x2 load2(const __half *p) {
  const float2 f = __half22float2(*(const __half2 *)p);
  return pair(f.x, f.y);
}
__device__ __forceinline__ f32x2 load2(const float *p) {
  const float2 f = *(const float2 *)p;
  return pair(f.x, f.y);
}
__device__ __forceinline__ uint32_t pack2(f32x2 x) {
  const float2 f = parts(x);
  return pack_bf16(f.x, f.y);
}

/* Eight lanes per row, 16 elements per lane in two runs of eight, such that a lane holds
 * both channels of its pairs: channels 8j .. and R/2 + 8j .. for the pairs
 * (i, i + R/2), 8j .. and 64 + 8j .. for (2i, 2i + 1) (INTER).  A warp takes four
 * neighbouring rows of a token at a time, of every 2^split, then its next token.
 *
 * HBM bounds it where there are many tokens, as long as enough is in flight and little
 * is computed per row.  A lane copies its 16-byte pieces of the rows ahead into slots of
 * its own in shared memory, DEPTH rows deep: no registers, no barriers.  The warp fetches
 * the table entries of its next token together while it computes this one, and the
 * positions of the one after it.  Two fp32 operations go in one instruction.
 *   30,000 tokens of 20 rows (323 MB) 55.6 us, 5.8 TB/s, 86% of the copy rate; 8,191
 * tokens 19.2; one token of 16 rows 1.8.  Steps: loads into registers a row ahead 69.9
 * and 21.7; the lanes fetching their own table entries 85; the axes in an indexed array
 * of the launch parameters 72; 16 lanes per row with one operation per instruction 78. */
constexpr int WARPS = 4, DEPTH = 3;

template <class T, bool INTER>
__global__ void __launch_bounds__(32 * WARPS, 16 / WARPS) norm_rope_kernel(const __grid_constant__ RowsParams p) {
  constexpr int PIECES = sizeof(T);                      // 16-byte pieces of a lane's 16 elements
  __shared__ uint4 rows_ahead[WARPS][DEPTH][PIECES][32];
  __shared__ float4 entries[WARPS][32];                  // [4][8 lanes] the entries of two pairs
  const int lane = threadIdx.x & 31, j = lane & 7;
  float4 *cs = entries[threadIdx.x >> 5];
  uint4 *ring = &rows_ahead[threadIdx.x >> 5][0][0][lane];   // this lane's slots: piece i of slot s at (s PIECES + i) 32
  const unsigned lanes = 0xffu << (lane & 24);
  const int R = p.rotary_dim, pairs = R / 2, split = p.split_log, step = 1 << split;   // split >= 2
  /* this lane's runs; lanes past R / 16 of the pairs (i, i + R / 2) hold what is not rotated */
  const int past = j - R / 16;
  const int e0 = INTER || past < 0 ? 8 * j : R + 8 * past;
  const int e1 = INTER ? D / 2 + 8 * j : past < 0 ? R / 2 + 8 * j : R + (D - R) / 2 + 8 * past;
  const bool rot_u = INTER ? e0 < R : past < 0, rot_v = INTER ? e1 < R : past < 0;
  /* items: a token's warps, 2^(split - 2) of them */
  const long long items = p.n_tokens << (split - 2), stride = (long long)gridDim.x * WARPS;
  long long item = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
  if (item >= items) return;
  const int first = (int)((unsigned)item << 2 & (step - 1)) + (lane >> 3);   // of the token's q, k and v rows, in this order
  const int h0 = p.set[0].heads, h1 = h0 + p.set[1].heads, h2 = h1 + p.set[2].heads;
  pdl_wait();
  pdl_trigger();
  auto position = [&](long long it, int i) {             // of pair lane + 32 i
    return it < items && lane + 32 * i < pairs
               ? p.positions[(long long)(p.axes[i] >> 2 * lane & 3) * p.n_tokens + (it >> (split - 2))]
               : -1;
  };
  auto entry = [&](int pos, int i) {
    return pos >= 0 && pos < p.table_len && lane + 32 * i < pairs ? p.table[(size_t)pos * pairs + lane + 32 * i]
                                                                  : make_float2(NAN, NAN);
  };
  int pos0 = position(item, 0), pos1 = position(item, 1);
  const T *q_src;
  const long long src_step = step * p.set[0].in_head, dst_step = step * p.set[0].out_head;
  auto rows_of = [&](long long tok) { q_src = (const T *)p.set[0].in + tok * p.set[0].in_token + first * p.set[0].in_head; };
  /* the rows ahead; most are query rows, a step apart, key and value rows are looked up */
  long long f_item = item;
  int f_row = first;
  rows_of(item >> (split - 2));
  auto fetch = [&](int slot) {
    if (f_row < h2 && f_item < items) {
      const T *src = q_src;
      q_src += src_step;
      if (f_row >= h0) {
        const long long tok = f_item >> (split - 2);
        src = f_row < h1 ? (const T *)p.set[1].in + tok * p.set[1].in_token + (f_row - h0) * p.set[1].in_head
                         : (const T *)p.set[2].in + tok * p.set[2].in_token + (f_row - h1) * p.set[2].in_head;
      }
#pragma unroll
      for (int i = 0; i < PIECES / 2; ++i) {
        cp_async16<PIECES == 4>(smem_u32(ring + (slot * PIECES + i) * 32), (const uint4 *)(src + e0) + i);
        cp_async16<PIECES == 4>(smem_u32(ring + (slot * PIECES + PIECES / 2 + i) * 32), (const uint4 *)(src + e1) + i);
      }
      f_row += step;
      if (f_row >= h2) {
        f_row = first;
        f_item += stride;
        rows_of(f_item >> (split - 2));
      }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < DEPTH; ++i) fetch(i);
  int slot = 0;
  float2 t0 = entry(pos0, 0), t1 = entry(pos1, 1);
  pos0 = position(item + stride, 0);
  pos1 = position(item + stride, 1);
  f32x2 cu[4], su[4], cv[4], sv[4], wu[4], wv[4];
  const float *have = nullptr;                           // whose weights are at hand
#pragma unroll 1
  for (; item < items; item += stride) {
    const long long tok = item >> (split - 2);
    __syncwarp();                                        // the entries before have been read
    auto put = [&](int q, float2 e) {                    // where lane j finds its eight pairs
      const int at = INTER ? (q / 32 * 2 + (q & 3) / 2) * 8 + (q & 31) / 4 : (q & 7) / 2 * 8 + q / 8;
      ((float2 *)cs)[at * 2 + (q & 1)] = e;
    };
    put(lane, t0);
    put(lane + 32, t1);
    __syncwarp();
    t0 = entry(pos0, 0);                                 // of the next token, and positions of the one after it
    t1 = entry(pos1, 1);
    pos0 = position(item + 2 * stride, 0);
    pos1 = position(item + 2 * stride, 1);
    /* (cos, sin) as the channels of runs u and v want them: INTER, word i: a pair's
     * cos twice, its -sin and sin; else the cosines and the sines of pairs 2i, 2i + 1 */
    if (rot_u) {                                           // rot_v: only with rot_u
      const float4 *e = cs + j;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (INTER) {                                       // word i of a run is a pair
          const float4 c = e[(i / 2) * 8], d = e[(i / 2 + 2) * 8];
          const float2 x = i & 1 ? make_float2(c.z, c.w) : make_float2(c.x, c.y);
          const float2 y = i & 1 ? make_float2(d.z, d.w) : make_float2(d.x, d.y);
          cu[i] = pair(x.x, x.x);
          su[i] = pair(-x.y, x.y);
          cv[i] = pair(y.x, y.x);
          sv[i] = pair(-y.y, y.y);
        } else {
          const float4 c = e[i * 8];
          cu[i] = cv[i] = pair(c.x, c.z);
          sv[i] = pair(c.y, c.w);
          su[i] = pair(-c.y, -c.w);
        }
      }
    }
    uint16_t *q_dst = p.set[0].out + tok * p.set[0].out_token + first * p.set[0].out_head;
#pragma unroll 1
    for (int row = first; row < h2; row += step, slot = (slot + 1) % DEPTH) {
      cp_async_wait<DEPTH - 1>();
      uint4 raw[PIECES];
#pragma unroll
      for (int i = 0; i < PIECES; ++i) raw[i] = ring[(slot * PIECES + i) * 32];
      auto two = [&](int run, int i) { return load2((const T *)raw + run * 8 + 2 * i); };
      uint4 u, v;
      uint32_t *ou = &u.x, *ov = &v.x;
      uint16_t *dst = q_dst;
      q_dst += dst_step;
      if (row >= h1) {                                     // a value row
        dst = p.set[2].out + tok * p.set[2].out_token + (row - h1) * p.set[2].out_head;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          ou[i] = pack2(two(0, i));
          ov[i] = pack2(two(1, i));
        }
      } else {
        const float *w = p.set[0].weight;
        if (row >= h0) {
          dst = p.set[1].out + tok * p.set[1].out_token + (row - h0) * p.set[1].out_head;
          w = p.set[1].weight;
        }
        f32x2 x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = two(0, i);
          y[i] = two(1, i);
        }
        if (w) {
          if (have != w) {
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
              const float4 a = *(const float4 *)(w + e0 + 2 * i), b = *(const float4 *)(w + e1 + 2 * i);
              wu[i] = pair(a.x, a.y);
              wu[i + 1] = pair(a.z, a.w);
              wv[i] = pair(b.x, b.y);
              wv[i + 1] = pair(b.z, b.w);
            }
            have = w;
          }
          f32x2 s2 = mul2(x[0], x[0]), t2 = mul2(y[0], y[0]);
#pragma unroll
          for (int i = 1; i < 4; ++i) {
            s2 = fma2(x[i], x[i], s2);
            t2 = fma2(y[i], y[i], t2);
          }
          const float2 s = parts(s2), t = parts(t2);
          float sum = (s.x + s.y) + (t.x + t.y);
#pragma unroll
          for (int o = 4; o; o >>= 1) sum += __shfl_xor_sync(lanes, sum, o);
          const float n = rsqrtf(sum * (1.f / D) + p.eps);
          const f32x2 f = pair(n, n);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[i] = mul2(mul2(x[i], f), wu[i]);
            y[i] = mul2(mul2(y[i], f), wv[i]);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f32x2 m = x[i], n = y[i];
          const float2 g = parts(x[i]), h = parts(y[i]);
          if (rot_u) m = fma2(INTER ? pair(g.y, g.x) : y[i], su[i], mul2(x[i], cu[i]));
          if (rot_v) n = fma2(INTER ? pair(h.y, h.x) : x[i], sv[i], mul2(y[i], cv[i]));
          ou[i] = pack2(m);
          ov[i] = pack2(n);
        }
      }
      *(uint4 *)(dst + e0) = u;
      *(uint4 *)(dst + e1) = v;
      fetch(slot);                                         // the slot has been read: its values are in the stores
    }
  }
}

/* Any layout that the call takes: 8-byte aligned rows, any multiple of 8 as
 * rotary_dim.  A warp per row, two pairs (or four elements) per lane.  8,191 tokens
 * of 20 rows 38 us, where 16-byte aligned rows take 17 in the kernel above (one set of
 * buffers, partly in L2). */
template <class T>
__global__ void __launch_bounds__(256) norm_rope_any_kernel(const __grid_constant__ RowsParams p, int inter) {
  pdl_wait();
  pdl_trigger();
  const int j = threadIdx.x & 31;
  const int all = p.set[0].heads + p.set[1].heads + p.set[2].heads;
  const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (unit >= p.n_tokens * all) return;
  const long long tok = unit / all;
  int k = 0, row = (int)(unit - tok * all);
  while (row >= p.set[k].heads) row -= p.set[k++].heads;
  const Rows &set = p.set[k];
  const int R = p.rotary_dim;
  const bool rot = 4 * j < R;
  const int e0 = inter || !rot ? 4 * j : 2 * j, e1 = inter || !rot ? e0 + 2 : R / 2 + 2 * j;
  const T *src = (const T *)set.in + tok * set.in_token + row * set.in_head;
  uint16_t *dst = set.out + tok * set.out_token + row * set.out_head;
  float2 x = parts(load2(src + e0)), y = parts(load2(src + e1));
  if (set.weight) {
    float sum = (x.x * x.x + x.y * x.y) + (y.x * y.x + y.y * y.y);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float n = rsqrtf(sum * (1.f / D) + p.eps);
    x = make_float2(x.x * n * set.weight[e0], x.y * n * set.weight[e0 + 1]);
    y = make_float2(y.x * n * set.weight[e1], y.y * n * set.weight[e1 + 1]);
  }
  if (rot && set.rotate) {
    float2 cs[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int q = 2 * j + i;
      const int pos = p.positions[(long long)((q < 32 ? p.axes[0] : p.axes[1]) >> 2 * (q & 31) & 3) * p.n_tokens + tok];
      cs[i] = make_float2(NAN, NAN);
      if (pos >= 0 && pos < p.table_len) cs[i] = p.table[(size_t)pos * (R / 2) + 2 * j + i];
    }
    const float2 u = x, v = y;
    if (inter) {
      x = make_float2(u.x * cs[0].x - u.y * cs[0].y, u.y * cs[0].x + u.x * cs[0].y);
      y = make_float2(v.x * cs[1].x - v.y * cs[1].y, v.y * cs[1].x + v.x * cs[1].y);
    } else {
      x = make_float2(u.x * cs[0].x - v.x * cs[0].y, u.y * cs[1].x - v.y * cs[1].y);
      y = make_float2(v.x * cs[0].x + u.x * cs[0].y, v.y * cs[1].x + u.y * cs[1].y);
    }
  }
  *(uint32_t *)(dst + e0) = pack_bf16(x.x, x.y);
  *(uint32_t *)(dst + e1) = pack_bf16(y.x, y.y);
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

constexpr int GRID = 152 * 16 / WARPS;   // blocks that run at once
constexpr int ROUND = GRID * WARPS * 4;   // units that run at once

static_assert(MD_MAX_AXES <= 4 && D / 2 <= 64, "an axis is two bits");

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
  const md_norm_rope_args &a = *args;
  if (a.n_tokens < 0 || a.num_q_heads < 0 || a.num_kv_heads < 0 || a.num_q_heads > 65535 || a.num_kv_heads > 65535 ||
      a.type < MD_TYPE_BF16 || a.type > MD_TYPE_F32 || a.rotary_dim < 0 || a.rotary_dim > D || a.rotary_dim % 8 ||
      !(a.eps >= 0.f))
    return MD_ERR_INVALID_ARG;
  const int values = a.v ? a.num_kv_heads : 0, rows = a.num_q_heads + a.num_kv_heads + values;
  if (a.n_tokens == 0 || rows == 0) return MD_OK;
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
  RowsParams p;
  memset(&p, 0, sizeof(p));
  if (a.rotary_dim > 0) {
    if (!a.table || !aligned(a.table, 16) || !a.positions || a.num_axes < 1 || a.num_axes > MD_MAX_AXES || a.table_len < 1)
      return MD_ERR_INVALID_ARG;
    for (int i = 0; a.axis_host && i < a.rotary_dim / 2; ++i) {
      if (a.axis_host[i] >= a.num_axes) return MD_ERR_INVALID_ARG;
      p.axes[i / 32] |= (unsigned long long)a.axis_host[i] << 2 * (i & 31);
    }
  }
  p.set[0] = {a.q, (uint16_t *)a.q_out, a.q_weight, a.q_token, a.q_head, a.q_out_token, a.q_out_head, a.num_q_heads, 1};
  p.set[1] = {a.k, (uint16_t *)a.k_out, a.k_weight, a.k_token, a.k_head, a.k_out_token, a.k_out_head, a.num_kv_heads, 1};
  p.set[2] = {a.v, (uint16_t *)a.v_out, nullptr, a.v_token, a.v_head, a.v_out_token, a.v_out_head, values, 0};
  p.table = (const float2 *)a.table;
  p.positions = a.positions;
  p.n_tokens = a.n_tokens;
  p.table_len = a.table_len;
  p.rotary_dim = a.rotary_dim;
  p.eps = a.eps;
  const cudaStream_t s = (cudaStream_t)a.stream;
  const int type = a.type;
  const bool inter = a.interleaved != 0;
  cudaError_t e;
  bool wide = a.rotary_dim % 16 == 0;
  for (const Rows &r : p.set) {
    const long long to = type == MD_TYPE_F32 ? 4 : 8;    // elements in 16 bytes
    if (r.heads)
      wide = wide && aligned(r.in, 16) && aligned(r.out, 16) && r.in_token % to == 0 && r.in_head % to == 0 &&
             r.out_token % 8 == 0 && r.out_head % 8 == 0;
  }
  if (wide) {
    /* a unit per row while one round of blocks has room for them */
    p.split_log = 2;
    while (1 << p.split_log < rows && (long long)a.n_tokens << (p.split_log + 1) <= ROUND) ++p.split_log;
    const long long blocks = (((long long)a.n_tokens << p.split_log) + 4 * WARPS - 1) / (4 * WARPS);
    auto launch = [&](auto plain, auto interleaved) {
      return launch_pdl(inter ? interleaved : plain, (int)(blocks < GRID ? blocks : GRID), 32 * WARPS, 0, s, p);
    };
    e = type == MD_TYPE_BF16  ? launch(norm_rope_kernel<__nv_bfloat16, false>, norm_rope_kernel<__nv_bfloat16, true>)
        : type == MD_TYPE_F16 ? launch(norm_rope_kernel<__half, false>, norm_rope_kernel<__half, true>)
                              : launch(norm_rope_kernel<float, false>, norm_rope_kernel<float, true>);
  } else {
    const long long blocks = ((long long)a.n_tokens * rows + 7) / 8;
    if (blocks >= (1LL << 31)) return MD_ERR_INVALID_ARG;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    auto launch = [&](auto kernel) { return cudaLaunchKernelEx(&cfg, kernel, p, (int)inter); };
    e = type == MD_TYPE_BF16  ? launch(norm_rope_any_kernel<__nv_bfloat16>)
        : type == MD_TYPE_F16 ? launch(norm_rope_any_kernel<__half>)
                              : launch(norm_rope_any_kernel<float>);
  }
  return e == cudaSuccess ? MD_OK : MD_ERR_CUDA;
}
