// Softmax attention, forward and backward, bf16 operands with 32-bit sums.
//
// Forward:   s = scale q k^T,  lse = log sum_j exp(s_j),  o = sum_j exp(s_j - lse) v_j.
// Backward:  p = exp(s - lse),  delta = sum_d do o,  ds = p (do v^T - delta),
//            dq = scale ds k,  dk = scale ds^T q,  dv = p^T do  (dk, dv summed over the query heads of a key head).
#include <math.h>

#include "operators.cuh"

namespace {

typedef __nv_bfloat16 bf16;

struct Sizes {
  int batch, tq, tk, heads, group, dim, causal;
  float scale;
  const int *q_lens, *kv_lens;
};

__device__ __forceinline__ int q_len(const Sizes &z, int b) { return z.q_lens ? min(max(z.q_lens[b], 0), z.tq) : z.tq; }
__device__ __forceinline__ int kv_len(const Sizes &z, int b) { return z.kv_lens ? min(max(z.kv_lens[b], 0), z.tk) : z.tk; }

// one warp per row; a lane holds elements lane, lane + 32, ... of the head
struct Row { float v[4]; };
__device__ __forceinline__ Row load_row(const bf16 *p, int dim) {
  Row r;
#pragma unroll
  for (int i = 0; i < 4; ++i) { const int c = (threadIdx.x & 31) + 32 * i; r.v[i] = c < dim ? __bfloat162float(p[c]) : 0.0f; }
  return r;
}
__device__ __forceinline__ void store_row(bf16 *p, int dim, const Row &r, float f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { const int c = (threadIdx.x & 31) + 32 * i; if (c < dim) p[c] = __float2bfloat16_rn(r.v[i] * f); }
}
__device__ __forceinline__ float dot(const Row &a, const Row &b) {
  return cdg_warp_sum(a.v[0] * b.v[0] + a.v[1] * b.v[1] + a.v[2] * b.v[2] + a.v[3] * b.v[3]);
}
__device__ __forceinline__ void axpy(Row &a, float f, const Row &b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) a.v[i] += f * b.v[i];
}

struct View { const bf16 *p; long long b, t, h; __device__ const bf16 *row(int bb, long long tt, int hh) const { return p + bb * b + tt * t + hh * h; } };
struct OutView { bf16 *p; long long b, t, h; __device__ bf16 *row(int bb, long long tt, int hh) const { return p + bb * b + tt * t + hh * h; } };

__global__ void __launch_bounds__(128) attn_forward_rows(Sizes z, View q, View k, View v, OutView o, float *lse) {
  const int i = blockIdx.x * 4 + (threadIdx.x >> 5), h = blockIdx.y, b = blockIdx.z;
  if (i >= z.tq) return;
  const int lq = q_len(z, b), lk = kv_len(z, b);
  int n = i < lq ? (z.causal ? min(lk, i + lk - lq + 1) : lk) : 0;
  Row acc = {}, qr = load_row(q.row(b, i, h), z.dim);
  float top = -INFINITY, sum = 0.0f;
  for (int j = 0; j < n; ++j) {
    const float s = z.scale * dot(qr, load_row(k.row(b, j, h / z.group), z.dim));
    const float nt = fmaxf(top, s), f = __expf(top - nt), p = __expf(s - nt);
    sum = sum * f + p;
#pragma unroll
    for (int c = 0; c < 4; ++c) acc.v[c] *= f;
    axpy(acc, p, load_row(v.row(b, j, h / z.group), z.dim));
    top = nt;
  }
  store_row(o.row(b, i, h), z.dim, acc, n > 0 ? 1.0f / sum : 0.0f);
  if ((threadIdx.x & 31) == 0) lse[((long long)b * z.heads + h) * z.tq + i] = n > 0 ? top + logf(sum) : -INFINITY;
}

__global__ void __launch_bounds__(128) attn_delta(Sizes z, View d_o, View o, float *delta) {
  const int i = blockIdx.x * 4 + (threadIdx.x >> 5), h = blockIdx.y, b = blockIdx.z;
  if (i >= z.tq) return;
  const float d = i < q_len(z, b) ? dot(load_row(d_o.row(b, i, h), z.dim), load_row(o.row(b, i, h), z.dim)) : 0.0f;
  if ((threadIdx.x & 31) == 0) delta[((long long)b * z.heads + h) * z.tq + i] = d;
}

__global__ void __launch_bounds__(128) attn_dq_rows(Sizes z, View q, View k, View v, View d_o, const float *lse,
                                                    const float *delta, OutView dq) {
  const int i = blockIdx.x * 4 + (threadIdx.x >> 5), h = blockIdx.y, b = blockIdx.z;
  if (i >= z.tq) return;
  const int lq = q_len(z, b), lk = kv_len(z, b);
  const int n = i < lq ? (z.causal ? min(lk, i + lk - lq + 1) : lk) : 0;
  Row acc = {}, qr = load_row(q.row(b, i, h), z.dim), dor = load_row(d_o.row(b, i, h), z.dim);
  const long long at = ((long long)b * z.heads + h) * z.tq + i;
  for (int j = 0; j < n; ++j) {
    const Row kr = load_row(k.row(b, j, h / z.group), z.dim);
    const float p = __expf(z.scale * dot(qr, kr) - lse[at]);
    const float dp = dot(dor, load_row(v.row(b, j, h / z.group), z.dim));
    axpy(acc, p * (dp - delta[at]), kr);
  }
  store_row(dq.row(b, i, h), z.dim, acc, z.scale);
}

__global__ void __launch_bounds__(128) attn_dkv_rows(Sizes z, View q, View k, View v, View d_o, const float *lse,
                                                     const float *delta, OutView dk, OutView dv) {
  const int j = blockIdx.x * 4 + (threadIdx.x >> 5), hk = blockIdx.y, b = blockIdx.z;
  if (j >= z.tk) return;
  const int lq = q_len(z, b), lk = kv_len(z, b);
  Row ak = {}, av = {}, kr = load_row(k.row(b, j, hk), z.dim), vr = load_row(v.row(b, j, hk), z.dim);
  const int first = j < lk ? (z.causal ? max(0, j - (lk - lq)) : 0) : lq;
  for (int h = hk * z.group; h < (hk + 1) * z.group; ++h)
    for (int i = first; i < lq; ++i) {
      const long long at = ((long long)b * z.heads + h) * z.tq + i;
      const Row qr = load_row(q.row(b, i, h), z.dim), dor = load_row(d_o.row(b, i, h), z.dim);
      const float p = __expf(z.scale * dot(qr, kr) - lse[at]);
      axpy(av, p, dor);
      axpy(ak, p * (dot(dor, vr) - delta[at]), qr);
    }
  store_row(dk.row(b, j, hk), z.dim, ak, z.scale);
  store_row(dv.row(b, j, hk), z.dim, av, 1.0f);
}

constexpr long long kMaxStride = 1ll << 38;   // elements; a tensor map holds byte strides below 2^40

// strides of a tensor that is read: multiples of 16 bytes, tokens and heads apart from each other
bool in_ok(const long long s[3], int tokens, int heads, int dim) {
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] % 8 != 0 || s[i] > kMaxStride) return false;
  return (tokens <= 1 || s[1] >= dim) && (heads <= 1 || s[2] >= dim);
}
// ... and of one that is written: no two heads' values on top of each other
bool out_ok(const long long s[3], int batch, int tokens, int heads, int dim) {
  if (!in_ok(s, tokens, heads, dim)) return false;
  long long ext[3] = {batch, tokens, heads}, str[3] = {s[0], s[1], s[2]}, span = dim;
  for (int round = 0; round < 3; ++round) {
    int at = -1;                                    // the axis with the smallest stride that is left
    for (int i = 0; i < 3; ++i)
      if (ext[i] > 1 && (at < 0 || str[i] < str[at])) at = i;
    if (at < 0) return true;
    if (str[at] < span) return false;
    span += (ext[at] - 1) * str[at];
    ext[at] = 1;
  }
  return true;
}

bool shape_ok(const cdgrab_attention_shape *s) {
  if (!s || s->batch < 0 || s->batch > 65535 || s->len_q < 0 || s->len_kv < 0 || s->heads < 1 || s->kv_heads < 1 ||
      s->heads > 65535 || s->heads % s->kv_heads != 0)
    return false;
  if (s->head_dim < 8 || s->head_dim > 128 || s->head_dim % 8 != 0 || (s->causal != 0 && s->causal != 1)) return false;
  return isfinite(s->scale);
}

Sizes sizes_of(const cdgrab_attention_shape *s, const int32_t *q_lens, const int32_t *kv_lens) {
  return Sizes{s->batch, s->len_q, s->len_kv, s->heads, s->heads / s->kv_heads, s->head_dim, s->causal, s->scale, q_lens, kv_lens};
}
View view(const void *p, const long long s[3]) { return View{(const bf16 *)p, s[0], s[1], s[2]}; }
OutView out_view(void *p, const long long s[3]) { return OutView{(bf16 *)p, s[0], s[1], s[2]}; }

}  // namespace

extern "C" int cdgrab_attention_forward(const cdgrab_attention_shape *s, const void *q, const void *k, const void *v,
                                        const int32_t *q_lens, const int32_t *kv_lens, void *o, float *lse,
                                        void *stream) {
  if (!shape_ok(s)) return CDGRAB_ERR_INVALID;
  if (s->batch == 0 || s->len_q == 0) return CDGRAB_OK;
  if (!q || !o || !lse || (s->len_kv > 0 && (!k || !v))) return CDGRAB_ERR_INVALID;
  if (!cdg_aligned(q, 16) || !cdg_aligned(k, 16) || !cdg_aligned(v, 16) || !cdg_aligned(o, 16) || !cdg_aligned(lse, 4) ||
      !cdg_aligned(q_lens, 4) || !cdg_aligned(kv_lens, 4))
    return CDGRAB_ERR_INVALID;
  if (!in_ok(s->q_stride, s->len_q, s->heads, s->head_dim) || !in_ok(s->k_stride, s->len_kv, s->kv_heads, s->head_dim) ||
      !in_ok(s->v_stride, s->len_kv, s->kv_heads, s->head_dim) ||
      !out_ok(s->o_stride, s->batch, s->len_q, s->heads, s->head_dim))
    return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  attn_forward_rows<<<dim3((s->len_q + 3) / 4, s->heads, s->batch), 128, 0, (cudaStream_t)stream>>>(
      sizes_of(s, q_lens, kv_lens), view(q, s->q_stride), view(k, s->k_stride), view(v, s->v_stride),
      out_view(o, s->o_stride), lse);
  return cdg_launch_rc();
}

extern "C" long long cdgrab_attention_workspace_bytes(const cdgrab_attention_shape *s) {
  if (!shape_ok(s)) return -1;
  return ((long long)s->batch * s->heads * s->len_q * 4 + 31) & ~15ll;
}

extern "C" int cdgrab_attention_backward(const cdgrab_attention_shape *s, const void *d_o, const void *q, const void *k,
                                         const void *v, const void *o, const float *lse, const int32_t *q_lens,
                                         const int32_t *kv_lens, void *dq, void *dk, void *dv, void *workspace,
                                         long long workspace_bytes, void *stream) {
  if (!shape_ok(s)) return CDGRAB_ERR_INVALID;
  if (s->batch == 0 || (s->len_q == 0 && s->len_kv == 0)) return CDGRAB_OK;
  if (s->len_q > 0 && (!q || !o || !d_o || !dq || !lse)) return CDGRAB_ERR_INVALID;
  if (s->len_kv > 0 && (!k || !v || !dk || !dv)) return CDGRAB_ERR_INVALID;
  const void *ptrs[] = {d_o, q, k, v, o, dq, dk, dv, workspace};
  for (const void *p : ptrs)
    if (!cdg_aligned(p, 16)) return CDGRAB_ERR_INVALID;
  if (!cdg_aligned(lse, 4) || !cdg_aligned(q_lens, 4) || !cdg_aligned(kv_lens, 4)) return CDGRAB_ERR_INVALID;
  const long long *qs[] = {s->q_stride, s->o_stride, s->do_stride}, *ks[] = {s->k_stride, s->v_stride};
  for (const long long *t : qs)
    if (!in_ok(t, s->len_q, s->heads, s->head_dim)) return CDGRAB_ERR_INVALID;
  for (const long long *t : ks)
    if (!in_ok(t, s->len_kv, s->kv_heads, s->head_dim)) return CDGRAB_ERR_INVALID;
  if (!out_ok(s->dq_stride, s->batch, s->len_q, s->heads, s->head_dim) ||
      !out_ok(s->dk_stride, s->batch, s->len_kv, s->kv_heads, s->head_dim) ||
      !out_ok(s->dv_stride, s->batch, s->len_kv, s->kv_heads, s->head_dim))
    return CDGRAB_ERR_INVALID;
  if (!workspace || workspace_bytes < cdgrab_attention_workspace_bytes(s)) return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const Sizes z = sizes_of(s, q_lens, kv_lens);
  float *delta = (float *)workspace;
  const View vq = view(q, s->q_stride), vk = view(k, s->k_stride), vv = view(v, s->v_stride), vdo = view(d_o, s->do_stride);
  const dim3 gq((s->len_q + 3) / 4, s->heads, s->batch), gk((s->len_kv + 3) / 4, s->kv_heads, s->batch);
  if (s->len_q > 0) {
    attn_delta<<<gq, 128, 0, st>>>(z, vdo, view(o, s->o_stride), delta);
    attn_dq_rows<<<gq, 128, 0, st>>>(z, vq, vk, vv, vdo, lse, delta, out_view(dq, s->dq_stride));
  }
  if (s->len_kv > 0)
    attn_dkv_rows<<<gk, 128, 0, st>>>(z, vq, vk, vv, vdo, lse, delta, out_view(dk, s->dk_stride), out_view(dv, s->dv_stride));
  return cdg_launch_rc();
}
