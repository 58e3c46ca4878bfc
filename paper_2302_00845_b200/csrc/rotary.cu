// Norms of queries and keys for each head and the rotation by the token's position, in one pass; and the backward pass,
// with the weights' gradients reduced per worker.
//
// Forward:   n = x rstd,  rstd = 1 / sqrt(sum x^2 / D + eps),  g = n w,  pairs of g turned by the angle t.
// Backward:  g' = the gradient turned by -t,  h = g' w,  dx = rstd (h - n (sum h n) / D),  dw = sum g' n.
// The angle of a far position is many turns: position x (frequency / 2 pi) is taken in 64 bits and only its fraction
// goes on in 32.
#include <cmath>

#include "operators.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxDim = 256, kMaxPairs = kMaxDim / 2;

// turns per position of each pair: base^(-2 i / rotary_dim) / (2 pi), 0 for the pairs that stay
struct Frequencies { double turns[kMaxPairs]; };

struct Args {
  const void *q, *k, *dq, *dk;
  void *qo, *ko;
  const float *qw, *kw;
  long long qs[3], ks[3], qos[3], kos[3], dqs[3], dks[3];
  const void *pos;
  int pos_bits;
  long long pos_stride;
  const int *lens;
  int len, heads, kv_heads, dim, rot, interleaved;
  float eps;
};

__device__ __forceinline__ long long position(const Args &a, long long b, int t) {
  if (!a.pos) return t;
  const long long at = b * a.pos_stride + t;
  return a.pos_bits == 64 ? static_cast<const long long *>(a.pos)[at] : static_cast<const int *>(a.pos)[at];
}
// where pair i's two values are
__device__ __forceinline__ int2 pair_at(const Args &a, int i) {
  const int half = a.rot / 2;
  if (i >= half) return make_int2(2 * i, 2 * i + 1);
  return a.interleaved ? make_int2(2 * i, 2 * i + 1) : make_int2(i, i + half);
}
__device__ __forceinline__ float2 turn(double turns) {
  const float f = (float)(turns - rint(turns));
  float s, c;
  sincospif(2.0f * f, &s, &c);
  return make_float2(c, s);
}

constexpr int kMine = kMaxPairs / 32;       // pairs to a lane

// a warp to a token, its heads in turn
template <typename T>
__global__ void __launch_bounds__(kThreads) rotary_forward_kernel(long long tokens, const __grid_constant__ Args a,
                                                                  const __grid_constant__ Frequencies f) {
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int lane = threadIdx.x & 31, pairs = a.dim / 2;
  for (long long tok = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5); tok < tokens; tok += (long long)gridDim.x * kWarps) {
    const long long b = tok / a.len;
    const int t = (int)(tok - b * a.len);
    const bool used = !a.lens || t < a.lens[b];
    const long long pos = position(a, b, t);
    float2 cs[kMine];
#pragma unroll
    for (int j = 0; j < kMine; ++j)
      if (lane + 32 * j < pairs) cs[j] = turn((double)pos * f.turns[lane + 32 * j]);
    for (int h = 0; h < a.heads + a.kv_heads; ++h) {
      const bool key = h >= a.heads;
      const int hh = key ? h - a.heads : h;
      const long long *is = key ? a.ks : a.qs, *os = key ? a.kos : a.qos;
      const T *x = static_cast<const T *>(key ? a.k : a.q) + b * is[0] + t * is[1] + hh * is[2];
      T *y = static_cast<T *>(key ? a.ko : a.qo) + b * os[0] + t * os[1] + hh * os[2];
      const float *w = key ? a.kw : a.qw;
      float2 v[kMine];
      float s = 0.0f;
#pragma unroll
      for (int j = 0; j < kMine; ++j) {
        v[j] = make_float2(0.0f, 0.0f);
        if (used && lane + 32 * j < pairs) {
          const int2 at = pair_at(a, lane + 32 * j);
          v[j] = make_float2(cdg_ld(x + at.x), cdg_ld(x + at.y));
        }
        s += v[j].x * v[j].x + v[j].y * v[j].y;
      }
      const float rstd = 1.0f / sqrtf(cdg_warp_sum(s) / (float)a.dim + a.eps);
      __syncwarp();
#pragma unroll
      for (int j = 0; j < kMine; ++j)
        if (lane + 32 * j < pairs) {
          const int2 at = pair_at(a, lane + 32 * j);
          const float p = v[j].x * rstd * (w ? w[at.x] : 1.0f), q = v[j].y * rstd * (w ? w[at.y] : 1.0f);
          y[at.x] = cdg_cast<T>(used ? p * cs[j].x - q * cs[j].y : 0.0f);
          y[at.y] = cdg_cast<T>(used ? p * cs[j].y + q * cs[j].x : 0.0f);
        }
    }
  }
}

// a block to a chunk (blockIdx.x) of a worker's tokens (blockIdx.y); its sums of g' n go to part[worker][chunk][2][dim]
template <typename T>
__global__ void __launch_bounds__(kThreads) rotary_backward_kernel(long long tokens, long long per, const __grid_constant__ Args a,
                                                                   const __grid_constant__ Frequencies f, float *part) {
  __shared__ float sums[kWarps][2][kMaxDim];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pairs = a.dim / 2;
  const long long first = (long long)blockIdx.y * tokens, end = first + min(tokens, (long long)(blockIdx.x + 1) * per);
  float2 dw[2][kMine] = {};
  for (long long tok = first + blockIdx.x * per + warp; tok < end; tok += kWarps) {
    const long long b = tok / a.len;
    const int t = (int)(tok - b * a.len);
    const bool used = !a.lens || t < a.lens[b];
    const long long pos = position(a, b, t);
    float2 cs[kMine];
#pragma unroll
    for (int j = 0; j < kMine; ++j)
      if (lane + 32 * j < pairs) cs[j] = turn((double)pos * f.turns[lane + 32 * j]);
#pragma unroll
    for (int key = 0; key < 2; ++key) {
      const long long *is = key ? a.ks : a.qs, *os = key ? a.kos : a.qos, *ds = key ? a.dks : a.dqs;
      const float *w = key ? a.kw : a.qw;
      for (int h = 0; h < (key ? a.kv_heads : a.heads); ++h) {
        const T *x = static_cast<const T *>(key ? a.k : a.q) + b * is[0] + t * is[1] + h * is[2];
        const T *dy = static_cast<const T *>(key ? a.dk : a.dq) + b * ds[0] + t * ds[1] + h * ds[2];
        T *y = static_cast<T *>(key ? a.ko : a.qo) + b * os[0] + t * os[1] + h * os[2];
        float2 v[kMine], g[kMine];
        float s = 0.0f, hn = 0.0f;
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
          v[j] = g[j] = make_float2(0.0f, 0.0f);
          if (used && lane + 32 * j < pairs) {
            const int2 at = pair_at(a, lane + 32 * j);
            v[j] = make_float2(cdg_ld(x + at.x), cdg_ld(x + at.y));
            const float p = cdg_ld(dy + at.x), q = cdg_ld(dy + at.y);
            g[j] = make_float2(p * cs[j].x + q * cs[j].y, q * cs[j].x - p * cs[j].y);
          }
          s += v[j].x * v[j].x + v[j].y * v[j].y;
        }
        const float rstd = 1.0f / sqrtf(cdg_warp_sum(s) / (float)a.dim + a.eps);
#pragma unroll
        for (int j = 0; j < kMine; ++j)
          if (used && lane + 32 * j < pairs) {
            const int2 at = pair_at(a, lane + 32 * j);
            v[j] = make_float2(v[j].x * rstd, v[j].y * rstd);
            dw[key][j].x += g[j].x * v[j].x;
            dw[key][j].y += g[j].y * v[j].y;
            g[j] = make_float2(g[j].x * (w ? w[at.x] : 1.0f), g[j].y * (w ? w[at.y] : 1.0f));
            hn += g[j].x * v[j].x + g[j].y * v[j].y;
          }
        hn = cdg_warp_sum(hn) / (float)a.dim;
#pragma unroll
        for (int j = 0; j < kMine; ++j)
          if (lane + 32 * j < pairs) {
            const int2 at = pair_at(a, lane + 32 * j);
            y[at.x] = cdg_cast<T>(used ? rstd * (g[j].x - v[j].x * hn) : 0.0f);
            y[at.y] = cdg_cast<T>(used ? rstd * (g[j].y - v[j].y * hn) : 0.0f);
          }
      }
    }
  }
  if (!part) return;
#pragma unroll
  for (int key = 0; key < 2; ++key)
#pragma unroll
    for (int j = 0; j < kMine; ++j)
      if (lane + 32 * j < pairs) {
        const int2 at = pair_at(a, lane + 32 * j);
        sums[warp][key][at.x] = dw[key][j].x;
        sums[warp][key][at.y] = dw[key][j].y;
      }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.dim; i += kThreads) {
    const int key = i >= a.dim, c = i - key * a.dim;
    float s = 0.0f;
    for (int o = 0; o < kWarps; ++o) s += sums[o][key][c];
    part[((long long)blockIdx.y * gridDim.x + blockIdx.x) * 2 * a.dim + i] = s;
  }
}

// the chunks' sums of one worker (blockIdx.x) added up in order
template <typename G>
__global__ void __launch_bounds__(kThreads) rotary_join_kernel(int chunks, int dim, const float *__restrict__ part, G *dqw, G *dkw,
                                                               long long ws) {
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  for (int i = threadIdx.x; i < 2 * dim; i += kThreads) {
    float s = 0.0f;
    for (int k = 0; k < chunks; ++k) s += part[((long long)blockIdx.x * chunks + k) * 2 * dim + i];
    G *out = i < dim ? dqw : dkw;
    if (out) out[(long long)blockIdx.x * ws + (i < dim ? i : i - dim)] = cdg_cast<G>(s);
  }
}

inline bool dtype_ok(int t) { return t == CDGRAB_F32 || t == CDGRAB_BF16; }

bool strides_ok(const long long (&s)[3], int len, int heads, int dim) {
  if (heads == 0) return true;
  for (long long v : s)
    if (v < 0 || v % 8 || v > (1ll << 40)) return false;
  return (len <= 1 || s[1] >= dim) && (heads <= 1 || s[2] >= dim);
}

bool shape_ok(const cdgrab_rotary_shape *s) {
  return s && s->batch >= 0 && s->len >= 0 && s->heads >= 0 && s->kv_heads >= 0 && s->heads <= 65535 && s->kv_heads <= 65535 &&
         s->head_dim >= 8 && s->head_dim <= kMaxDim && s->head_dim % 8 == 0 && s->rotary_dim >= 0 && s->rotary_dim <= s->head_dim &&
         s->rotary_dim % 8 == 0 && (s->interleaved == 0 || s->interleaved == 1) && dtype_ok(s->dtype) && s->base > 0.0 &&
         std::isfinite(s->base) && s->eps >= 0.0f && std::isfinite(s->eps) && s->reserved == 0 && (long long)s->batch * s->len < (1ll << 31) &&
         (long long)(s->heads + s->kv_heads) * s->head_dim < (1ll << 31);
}

int chunks_of(long long tokens, int m) {
  const long long most = 148 * 8 / m, fit = (tokens + kWarps - 1) / kWarps, c = most < fit ? most : fit;
  return (int)(c < 1 ? 1 : c);
}

void fill(const cdgrab_rotary_shape *s, Args &a, Frequencies &f) {
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = s->q_stride[i]; a.ks[i] = s->k_stride[i]; a.qos[i] = s->q_out_stride[i]; a.kos[i] = s->k_out_stride[i];
    a.dqs[i] = s->dq_stride[i]; a.dks[i] = s->dk_stride[i];
  }
  a.len = s->len; a.heads = s->heads; a.kv_heads = s->kv_heads; a.dim = s->head_dim; a.rot = s->rotary_dim;
  a.interleaved = s->interleaved; a.eps = s->eps;
  // (a power for each pair costs more than the launch: each thread keeps its last table)
  static thread_local struct { double base; int rot; Frequencies f; } last = {};
  if (last.base != s->base || last.rot != s->rotary_dim) {
    for (int i = 0; i < kMaxPairs; ++i)
      last.f.turns[i] = 2 * i < s->rotary_dim ? std::pow(s->base, -2.0 * i / s->rotary_dim) / (2.0 * M_PI) : 0.0;
    last.base = s->base;
    last.rot = s->rotary_dim;
  }
  f = last.f;
}

// the checks that both directions share; backward: with the gradients
bool call_ok(const cdgrab_rotary_shape *s, const Args &a, bool backward) {
  if (!strides_ok(s->q_stride, s->len, s->heads, s->head_dim) || !strides_ok(s->k_stride, s->len, s->kv_heads, s->head_dim) ||
      !strides_ok(s->q_out_stride, s->len, s->heads, s->head_dim) || !strides_ok(s->k_out_stride, s->len, s->kv_heads, s->head_dim))
    return false;
  if (backward && (!strides_ok(s->dq_stride, s->len, s->heads, s->head_dim) || !strides_ok(s->dk_stride, s->len, s->kv_heads, s->head_dim)))
    return false;
  if (s->heads > 0 && (!a.q || !a.qo || (backward && !a.dq))) return false;
  if (s->kv_heads > 0 && (!a.k || !a.ko || (backward && !a.dk))) return false;
  for (const void *p : {a.q, a.k, a.dq, a.dk, (const void *)a.qo, (const void *)a.ko})
    if (!cdg_aligned(p, 16)) return false;
  if (!cdg_aligned(a.qw, 4) || !cdg_aligned(a.kw, 4) || !cdg_aligned(a.lens, 4)) return false;
  return !a.pos || ((a.pos_bits == 32 || a.pos_bits == 64) && a.pos_stride >= 0 && cdg_aligned(a.pos, a.pos_bits / 8));
}

}  // namespace

extern "C" int cdgrab_rotary_forward(const cdgrab_rotary_shape *s, const void *q, const void *k, const float *qw, const float *kw,
                                     const void *pos, int pos_bits, long long pos_stride, const int32_t *lens, void *qo, void *ko,
                                     void *stream) {
  if (!shape_ok(s)) return CDGRAB_ERR_INVALID;
  if (s->batch == 0 || s->len == 0 || s->heads + s->kv_heads == 0) return CDGRAB_OK;
  Args a = {q, k, nullptr, nullptr, qo, ko, qw, kw};
  a.pos = pos; a.pos_bits = pos_bits; a.pos_stride = pos_stride; a.lens = lens;
  if (!call_ok(s, a, false)) return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  Frequencies f;
  fill(s, a, f);
  const long long tokens = (long long)s->batch * s->len, blocks = (tokens + kWarps - 1) / kWarps, most = (long long)dev->sms * 8;
  const dim3 grid((unsigned)(blocks < most ? blocks : most));
  cudaStream_t st = (cudaStream_t)stream;
  return cdg_launch_rc(s->dtype == CDGRAB_F32 ? cdg_ops_launch(rotary_forward_kernel<float>, grid, kThreads, 0, st, tokens, a, f)
                                              : cdg_ops_launch(rotary_forward_kernel<__nv_bfloat16>, grid, kThreads, 0, st, tokens, a, f));
}

extern "C" long long cdgrab_rotary_workspace_bytes(const cdgrab_rotary_shape *s, int m) {
  if (!shape_ok(s) || m < 1 || m > 65535 || s->batch % m) return -1;
  return 8ll * m * chunks_of((long long)s->batch / m * s->len, m) * s->head_dim;
}

extern "C" int cdgrab_rotary_backward(const cdgrab_rotary_shape *s, int m, const void *dq, const void *dk, const void *q, const void *k,
                                      const float *qw, const float *kw, const void *pos, int pos_bits, long long pos_stride,
                                      const int32_t *lens, void *qo, void *ko, int grad_dtype, void *dqw, void *dkw,
                                      long long worker_stride, void *workspace, long long workspace_bytes, void *stream) {
  const long long need = cdgrab_rotary_workspace_bytes(s, m);
  if (need < 0 || !dtype_ok(grad_dtype)) return CDGRAB_ERR_INVALID;
  Args a = {q, k, dq, dk, qo, ko, qw, kw};
  a.pos = pos; a.pos_bits = pos_bits; a.pos_stride = pos_stride; a.lens = lens;
  const long long tokens = (long long)s->batch / m * s->len;
  if (tokens > 0 && !call_ok(s, a, true)) return CDGRAB_ERR_INVALID;
  const int ge = grad_dtype == CDGRAB_F32 ? 4 : 2;
  if (((dqw || dkw) && m > 1 && worker_stride < s->head_dim) || !cdg_aligned(dqw, ge) || !cdg_aligned(dkw, ge)) return CDGRAB_ERR_INVALID;
  if (!workspace || workspace_bytes < need || !cdg_aligned(workspace, 16)) return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  Frequencies f;
  fill(s, a, f);
  const int chunks = chunks_of(tokens, m);
  const dim3 grid(chunks, m);
  cudaStream_t st = (cudaStream_t)stream;
  float *part = dqw || dkw ? static_cast<float *>(workspace) : nullptr;
  const long long per = (tokens + chunks - 1) / chunks;
  int rc = cdg_launch_rc(s->dtype == CDGRAB_F32 ? cdg_ops_launch(rotary_backward_kernel<float>, grid, kThreads, 0, st, tokens, per, a, f, part)
                                                : cdg_ops_launch(rotary_backward_kernel<__nv_bfloat16>, grid, kThreads, 0, st, tokens, per, a, f, part));
  if (rc == CDGRAB_OK && part)
    rc = cdg_launch_rc(grad_dtype == CDGRAB_F32
                           ? cdg_ops_launch(rotary_join_kernel<float>, dim3(m), kThreads, 0, st, chunks, s->head_dim, part, (float *)dqw, (float *)dkw, worker_stride)
                           : cdg_ops_launch(rotary_join_kernel<__nv_bfloat16>, dim3(m), kThreads, 0, st, chunks, s->head_dim, part,
                                            (__nv_bfloat16 *)dqw, (__nv_bfloat16 *)dkw, worker_stride));
  return rc;
}
