// The orthogonalised update: Newton-Schulz products that drive a matrix's singular values to one.
//
//   X = G / (|G|_F + eps);  steps times:  A = X X^T,  B = b A + c A A,  X <- a X + B X
// on the transposed matrix where G has more rows than columns (m <= n below).
#include <math.h>

#include "operators.cuh"

namespace {

constexpr int kTile = 64, kDepth = 16, kNormBlocks = 64;

template <typename T>
__global__ void __launch_bounds__(256) orth_sumsq(const T *g, long long gb, long long gs, int rows, int cols,
                                                  double *part) {
  __shared__ double sm[256];
  const T *p = g + blockIdx.y * gb;
  double s = 0.0;
  for (int r = blockIdx.x; r < rows; r += gridDim.x)
    for (int c = threadIdx.x; c < cols; c += 256) { const double v = cdg_ld(p + r * gs + c); s += v * v; }
  sm[threadIdx.x] = s;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (threadIdx.x < o) sm[threadIdx.x] += sm[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) part[blockIdx.y * gridDim.x + blockIdx.x] = sm[0];
}

// x[m][n] = G (or its transpose) / (norm + eps)
template <typename T>
__global__ void __launch_bounds__(256) orth_start(const T *g, long long gb, long long gs, int m, int n, int tall,
                                                  const double *part, float eps, float *x) {
  double t = 0.0;
  for (int i = 0; i < kNormBlocks; ++i) t += part[blockIdx.y * kNormBlocks + i];
  const float f = (float)(1.0 / (sqrt(t) + (double)eps));
  for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < (long long)m * n; e += (long long)gridDim.x * 256) {
    const long long r = e / n, c = e % n;
    x[blockIdx.y * (long long)m * n + e] = f * cdg_ld(g + blockIdx.y * gb + (tall ? c * gs + r : r * gs + c));
  }
}

// C[m][n] = alpha A op(B) + beta D, row-major, op(B) = B^T (B is [n][k]) or B ([k][n])
template <bool TB>
__global__ void __launch_bounds__(256) orth_product(int m, int n, int k, float alpha, const float *A, const float *B,
                                                    float beta, const float *D, float *C) {
  __shared__ float sa[kDepth][kTile + 1], sb[kDepth][kTile + 1];
  A += (long long)blockIdx.z * m * k; B += (long long)blockIdx.z * n * k;
  D += (long long)blockIdx.z * m * n; C += (long long)blockIdx.z * m * n;
  const int i0 = blockIdx.y * kTile, j0 = blockIdx.x * kTile, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {};
  for (int k0 = 0; k0 < k; k0 += kDepth) {
    for (int e = threadIdx.x; e < kTile * kDepth; e += 256) {
      int r = e / kDepth, kk = e % kDepth;
      sa[kk][r] = i0 + r < m && k0 + kk < k ? A[(long long)(i0 + r) * k + k0 + kk] : 0.0f;
      if (TB) {
        sb[kk][r] = j0 + r < n && k0 + kk < k ? B[(long long)(j0 + r) * k + k0 + kk] : 0.0f;
      } else {
        r = e % kTile; kk = e / kTile;
        sb[kk][r] = j0 + r < n && k0 + kk < k ? B[(long long)(k0 + kk) * n + j0 + r] : 0.0f;
      }
    }
    __syncthreads();
    for (int kk = 0; kk < kDepth; ++kk)
      for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) acc[a][b] += sa[kk][ty + 16 * a] * sb[kk][tx + 16 * b];
    __syncthreads();
  }
  for (int a = 0; a < 4; ++a)
    for (int b = 0; b < 4; ++b) {
      const int i = i0 + ty + 16 * a, j = j0 + tx + 16 * b;
      if (i < m && j < n) {
        const long long at = (long long)i * n + j;
        C[at] = alpha * acc[a][b] + (beta != 0.0f ? beta * D[at] : 0.0f);
      }
    }
}

__global__ void __launch_bounds__(256) orth_finish(int m, int n, int tall, const float *x, __nv_bfloat16 *o,
                                                   long long ob, long long os) {
  for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < (long long)m * n; e += (long long)gridDim.x * 256) {
    const long long r = e / n, c = e % n;
    o[blockIdx.y * ob + (tall ? c * os + r : r * os + c)] = __float2bfloat16_rn(x[blockIdx.y * (long long)m * n + e]);
  }
}

inline long long up16(long long v) { return (v + 15) & ~15ll; }

}  // namespace

extern "C" long long cdgrab_orthogonalise_workspace_bytes(int batch, int rows, int cols) {
  if (batch < 0 || batch > 65535 || rows < 0 || cols < 0 || rows > (1 << 20) || cols > (1 << 20)) return -1;
  const long long m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
  return up16(8ll * batch * kNormBlocks) + 2 * up16(4 * batch * m * n) + 2 * up16(4 * batch * m * m) + 16;
}

extern "C" int cdgrab_orthogonalise(int batch, int rows, int cols, int dtype, const void *g, long long gb, long long gs,
                                    int steps, const float *coeffs, float eps, void *o, long long ob, long long os,
                                    void *workspace, long long workspace_bytes, void *stream) {
  const long long need = cdgrab_orthogonalise_workspace_bytes(batch, rows, cols);
  if (need < 0 || steps < 1 || steps > 64 || !coeffs || !(eps >= 0.0f) || (dtype != CDGRAB_F32 && dtype != CDGRAB_BF16))
    return CDGRAB_ERR_INVALID;
  if (!isfinite(coeffs[0]) || !isfinite(coeffs[1]) || !isfinite(coeffs[2])) return CDGRAB_ERR_INVALID;
  if (batch == 0 || rows == 0 || cols == 0) return CDGRAB_OK;
  if (!g || !o || !workspace || workspace_bytes < need || !cdg_aligned(workspace, 16) || gs < cols || os < cols ||
      (batch > 1 && (gb < 0 || ob < (long long)(rows - 1) * os + cols)))
    return CDGRAB_ERR_INVALID;
  if (!cdg_aligned(g, dtype == CDGRAB_F32 ? 4 : 2) || !cdg_aligned(o, 2)) return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const int tall = rows > cols, m = tall ? cols : rows, n = tall ? rows : cols;
  char *p = (char *)workspace;
  double *part = (double *)p; p += up16(8ll * batch * kNormBlocks);
  float *x = (float *)p; p += up16(4ll * batch * m * n);
  float *y = (float *)p; p += up16(4ll * batch * m * n);
  float *A = (float *)p; p += up16(4ll * batch * m * m);
  float *B = (float *)p;
  const dim3 gn(kNormBlocks, batch), gx(2 * dev->sms, batch);
  const dim3 gm((m + kTile - 1) / kTile, (m + kTile - 1) / kTile, batch), gx2((n + kTile - 1) / kTile, (m + kTile - 1) / kTile, batch);
  if (dtype == CDGRAB_F32) {
    orth_sumsq<<<gn, 256, 0, st>>>((const float *)g, gb, gs, rows, cols, part);
    orth_start<<<gx, 256, 0, st>>>((const float *)g, gb, gs, m, n, tall, part, eps, x);
  } else {
    orth_sumsq<<<gn, 256, 0, st>>>((const __nv_bfloat16 *)g, gb, gs, rows, cols, part);
    orth_start<<<gx, 256, 0, st>>>((const __nv_bfloat16 *)g, gb, gs, m, n, tall, part, eps, x);
  }
  for (int i = 0; i < steps; ++i) {
    orth_product<true><<<gm, 256, 0, st>>>(m, m, n, 1.0f, x, x, 0.0f, x, A);
    orth_product<true><<<gm, 256, 0, st>>>(m, m, m, coeffs[2], A, A, coeffs[1], A, B);
    orth_product<false><<<gx2, 256, 0, st>>>(m, n, m, 1.0f, B, x, coeffs[0], x, y);
    float *t = x; x = y; y = t;
  }
  orth_finish<<<gx, 256, 0, st>>>(m, n, tall, x, (__nv_bfloat16 *)o, ob, os);
  return cdg_launch_rc();
}
