// Layer normalisation, forward and backward, with the weight's gradient reduced per worker.
//
// Forward:   mean = sum x / C,  var = sum (x - mean)^2 / C,  y = (x - mean) / sqrt(var + eps) * w + b.
// Backward:  n = (x - mean) rstd,  g = dy w,  dx = rstd (g - sum g / C - n (sum g n) / C),
//            dw = sum over a worker's rows of dy n,  db = the same of dy.
#include "operators.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// sum of a and b over the block, the same value in every thread
__device__ __forceinline__ float2 block_sum(float a, float b, float2 *sm) {
  a = cdg_warp_sum(a);
  b = cdg_warp_sum(b);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = make_float2(a, b);
  __syncthreads();
  float2 t = sm[0];
  for (int w = 1; w < (int)(blockDim.x >> 5); ++w) { t.x += sm[w].x; t.y += sm[w].y; }
  return t;
}

// one block per row, three passes over it
template <typename T>
__global__ void __launch_bounds__(kThreads) ln_forward_long(int cols, const T *__restrict__ x, long long xs,
                                                            const float *__restrict__ w, const float *__restrict__ b,
                                                            float eps, T *y, long long ys, float *mean_out,
                                                            float *rstd_out) {
  __shared__ float2 sm[kWarps];
  const T *xr = x + (long long)blockIdx.x * xs;
  T *yr = y + (long long)blockIdx.x * ys;
  const float inv = 1.0f / (float)cols;
  float s = 0.0f;
  for (int c = threadIdx.x; c < cols; c += kThreads) s += cdg_ld(xr + c);
  const float mean = block_sum(s, 0.0f, sm).x * inv;
  s = 0.0f;
  for (int c = threadIdx.x; c < cols; c += kThreads) { const float d = cdg_ld(xr + c) - mean; s += d * d; }
  const float rstd = 1.0f / sqrtf(block_sum(s, 0.0f, sm).x * inv + eps);
  for (int c = threadIdx.x; c < cols; c += kThreads) {
    const float n = (cdg_ld(xr + c) - mean) * rstd;
    yr[c] = cdg_cast<T>(n * (w ? w[c] : 1.0f) + (b ? b[c] : 0.0f));
  }
  if (threadIdx.x == 0) {
    if (mean_out) mean_out[blockIdx.x] = mean;
    if (rstd_out) rstd_out[blockIdx.x] = rstd;
  }
}

// the worker's sums of dy n and dy, one thread per column (before dx: it may overwrite dy or x)
template <typename T, typename G>
__global__ void __launch_bounds__(kThreads) ln_backward_columns(long long rows, int cols, const T *__restrict__ dy,
                                                                long long dys, const T *__restrict__ x, long long xs,
                                                                const float *__restrict__ mean,
                                                                const float *__restrict__ rstd, G *dw, G *db,
                                                                long long ws) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= cols) return;
  const long long r0 = (long long)blockIdx.y * rows;
  float sw = 0.0f, sb = 0.0f;
  for (long long r = r0; r < r0 + rows; ++r) {
    const float d = cdg_ld(dy + r * dys + c);
    sw += d * ((cdg_ld(x + r * xs + c) - mean[r]) * rstd[r]);
    sb += d;
  }
  if (dw) dw[(long long)blockIdx.y * ws + c] = cdg_cast<G>(sw);
  if (db) db[(long long)blockIdx.y * ws + c] = cdg_cast<G>(sb);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) ln_backward_long(int cols, const T *dy, long long dys, const T *x,
                                                             long long xs, const float *__restrict__ w,
                                                             const float *__restrict__ mean,
                                                             const float *__restrict__ rstd, T *dx, long long dxs) {
  __shared__ float2 sm[kWarps];
  const long long r = blockIdx.x;
  const T *dyr = dy + r * dys, *xr = x + r * xs;
  T *dxr = dx + r * dxs;
  const float mu = mean[r], rs = rstd[r], inv = 1.0f / (float)cols;
  float s1 = 0.0f, s2 = 0.0f;
  for (int c = threadIdx.x; c < cols; c += kThreads) {
    const float g = cdg_ld(dyr + c) * (w ? w[c] : 1.0f);
    s1 += g;
    s2 += g * ((cdg_ld(xr + c) - mu) * rs);
  }
  const float2 t = block_sum(s1, s2, sm);
  for (int c = threadIdx.x; c < cols; c += kThreads) {
    const float g = cdg_ld(dyr + c) * (w ? w[c] : 1.0f);
    const float n = (cdg_ld(xr + c) - mu) * rs;
    dxr[c] = cdg_cast<T>(rs * (g - t.x * inv - n * (t.y * inv)));
  }
}

inline bool dtype_ok(int t) { return t == CDGRAB_F32 || t == CDGRAB_BF16; }

}  // namespace

extern "C" int cdgrab_layer_norm_forward(long long rows, int cols, int dtype, const void *x, long long xs,
                                         const float *w, const float *b, float eps, void *y, long long ys,
                                         float *mean, float *rstd, void *stream) {
  if (rows < 0 || rows >= (1ll << 31) || cols < 1 || !dtype_ok(dtype) || !(eps >= 0.0f)) return CDGRAB_ERR_INVALID;
  if (rows == 0) return CDGRAB_OK;
  if (!x || !y || xs < cols || ys < cols) return CDGRAB_ERR_INVALID;
  const size_t e = dtype == CDGRAB_F32 ? 4 : 2;
  if (!cdg_aligned(x, e) || !cdg_aligned(y, e) || !cdg_aligned(w, 4) || !cdg_aligned(b, 4) || !cdg_aligned(mean, 4) ||
      !cdg_aligned(rstd, 4))
    return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == CDGRAB_F32)
    ln_forward_long<<<(unsigned)rows, kThreads, 0, st>>>(cols, (const float *)x, xs, w, b, eps, (float *)y, ys, mean, rstd);
  else
    ln_forward_long<<<(unsigned)rows, kThreads, 0, st>>>(cols, (const __nv_bfloat16 *)x, xs, w, b, eps,
                                                         (__nv_bfloat16 *)y, ys, mean, rstd);
  return cdg_launch_rc();
}

extern "C" long long cdgrab_layer_norm_workspace_bytes(int m, long long rows, int cols) {
  if (m < 1 || m > 65535 || rows < 0 || cols < 1 || (rows > 0 && m >= (1ll << 31) / rows)) return -1;
  return 16;
}

template <typename T, typename G>
static int ln_backward(int m, long long rows, int cols, const void *dy, long long dys, const void *x, long long xs,
                       const float *w, const float *mean, const float *rstd, void *dx, long long dxs, void *dw,
                       void *db, long long ws, cudaStream_t st) {
  if (dw || db)
    ln_backward_columns<T, G><<<dim3((cols + kThreads - 1) / kThreads, m), kThreads, 0, st>>>(
        rows, cols, (const T *)dy, dys, (const T *)x, xs, mean, rstd, (G *)dw, (G *)db, ws);
  if (dx && rows)
    ln_backward_long<T><<<(unsigned)(m * rows), kThreads, 0, st>>>(cols, (const T *)dy, dys, (const T *)x, xs, w,
                                                                   mean, rstd, (T *)dx, dxs);
  return cdg_launch_rc();
}

extern "C" int cdgrab_layer_norm_backward(int m, long long rows, int cols, int dtype, const void *dy, long long dys,
                                          const void *x, long long xs, const float *w, const float *mean,
                                          const float *rstd, void *dx, long long dxs, int grad_dtype, void *dw,
                                          void *db, long long ws, void *workspace, long long workspace_bytes,
                                          void *stream) {
  const long long need = cdgrab_layer_norm_workspace_bytes(m, rows, cols);
  if (need < 0 || !dtype_ok(dtype) || !dtype_ok(grad_dtype)) return CDGRAB_ERR_INVALID;
  if (rows > 0 && (!dy || !x || !mean || !rstd || dys < cols || xs < cols || (dx && dxs < cols))) return CDGRAB_ERR_INVALID;
  if ((dw || db) && m > 1 && ws < cols) return CDGRAB_ERR_INVALID;
  if (!workspace || workspace_bytes < need || !cdg_aligned(workspace, 16)) return CDGRAB_ERR_INVALID;
  const size_t e = dtype == CDGRAB_F32 ? 4 : 2, ge = grad_dtype == CDGRAB_F32 ? 4 : 2;
  if (!cdg_aligned(dy, e) || !cdg_aligned(x, e) || !cdg_aligned(dx, e) || !cdg_aligned(dw, ge) || !cdg_aligned(db, ge) ||
      !cdg_aligned(w, 4) || !cdg_aligned(mean, 4) || !cdg_aligned(rstd, 4))
    return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == CDGRAB_F32)
    return grad_dtype == CDGRAB_F32 ? ln_backward<float, float>(m, rows, cols, dy, dys, x, xs, w, mean, rstd, dx, dxs, dw, db, ws, st)
                                    : ln_backward<float, __nv_bfloat16>(m, rows, cols, dy, dys, x, xs, w, mean, rstd, dx, dxs, dw, db, ws, st);
  return grad_dtype == CDGRAB_F32 ? ln_backward<__nv_bfloat16, float>(m, rows, cols, dy, dys, x, xs, w, mean, rstd, dx, dxs, dw, db, ws, st)
                                  : ln_backward<__nv_bfloat16, __nv_bfloat16>(m, rows, cols, dy, dys, x, xs, w, mean, rstd, dx, dxs, dw, db, ws, st);
}
