// Embedding lookup and its gradient, reduced per worker into the gather buffer.
//
//   y[r] = scale table[t_r];   dtable[i][v] = scale sum of dy[r] over worker i's rows r with t_r = v.
#include <cmath>

#include "operators.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

struct Tokens {
  const void *p;
  int bits;
  long long stride, length, padding;
  int vocab;
  // token j of row g of the tokens
  __device__ __forceinline__ long long at(long long g, long long j) const {
    return bits == 64 ? static_cast<const long long *>(p)[g * stride + j] : static_cast<const int *>(p)[g * stride + j];
  }
  __device__ __forceinline__ bool valid(long long t) const { return t >= 0 && t < vocab && t != padding; }
};

template <typename T, typename R>
__global__ void __launch_bounds__(kThreads) lookup_kernel(long long rows, int cols, Tokens tok, float scale, const T *__restrict__ table,
                                                          long long ts, R *__restrict__ y, long long ys, int *status) {
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int lane = threadIdx.x & 31;
  for (long long r = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5); r < rows; r += (long long)gridDim.x * kWarps) {
    const long long g = r / tok.length, t = tok.at(g, r - g * tok.length);
    const bool valid = tok.valid(t);
    if (!valid && t != tok.padding && lane == 0) atomicOr(status, CDG_ST_INDEX);
    for (int c = lane; c < cols; c += 32) y[r * ys + c] = cdg_cast<R>(valid ? cdg_ld(table + t * ts + c) * scale : 0.0f);
  }
}

// a warp to a worker's row of the table: all of the worker's tokens are looked through
template <typename T, typename G>
__global__ void __launch_bounds__(kThreads) gradient_kernel(long long groups, int cols, Tokens tok, float scale, const T *__restrict__ dy,
                                                            long long dys, G *dtable, long long ws, long long rs, int accumulate,
                                                            int *status) {
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int lane = threadIdx.x & 31;
  const long long v = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5), w = blockIdx.y, n = groups * tok.length;
  if (v >= tok.vocab) return;
  G *out = dtable + w * ws + v * rs;
  for (long long c0 = 0; c0 < cols; c0 += 32) {
    const long long c = c0 + lane;
    float s = 0.0f;
    bool any = false;
    for (long long j = 0; j < n; ++j) {
      const long long t = tok.at(w * groups + j / tok.length, j % tok.length);
      if (v == 0 && !tok.valid(t) && t != tok.padding) atomicOr(status, CDG_ST_INDEX);
      if (t != v || !tok.valid(t)) continue;
      any = true;
      if (c < cols) s += cdg_ld(dy + (w * n + j) * dys + c);
    }
    if (c < cols && (any || !accumulate)) out[c] = cdg_cast<G>(accumulate ? cdg_ld(out + c) + s * scale : s * scale);
  }
}

inline bool dtype_ok(int t) { return t == CDGRAB_F32 || t == CDGRAB_BF16; }
inline int size_of(int dtype) { return dtype == CDGRAB_F32 ? 4 : 2; }

}  // namespace

extern "C" int cdgrab_embedding_forward(long long groups, long long length, int cols, int vocab, int token_bits, const void *tokens,
                                        long long token_stride, long long padding, float scale, int dtype, const void *table,
                                        long long table_stride, int out_dtype, void *y, long long y_stride, void *stream) {
  if (groups < 0 || length < 0 || (length > 0 && groups >= ((1ll << 31) + length - 1) / length) || cols < 1 || vocab < 1 ||
      (token_bits != 32 && token_bits != 64) || !std::isfinite(scale) || !dtype_ok(dtype) || !dtype_ok(out_dtype))
    return CDGRAB_ERR_INVALID;
  if (groups == 0 || length == 0) return CDGRAB_OK;
  if (!tokens || !table || !y || (groups > 1 && token_stride < length) || (vocab > 1 && table_stride < cols) || y_stride < cols ||
      !cdg_aligned(tokens, token_bits / 8) || !cdg_aligned(table, size_of(dtype)) || !cdg_aligned(y, size_of(out_dtype)))
    return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  const long long rows = groups * length, blocks = (rows + kWarps - 1) / kWarps, most = (long long)dev->sms * 8;
  const Tokens tok = {tokens, token_bits, token_stride, length, padding, vocab};
  const dim3 grid((unsigned)(blocks < most ? blocks : most));
  cudaStream_t st = (cudaStream_t)stream;
  auto go = [&](auto t, auto r) {
    using T = decltype(t);
    using R = decltype(r);
    return cdg_launch_rc(cdg_ops_launch(lookup_kernel<T, R>, grid, kThreads, 0, st, rows, cols, tok, scale, (const T *)table, table_stride,
                                        (R *)y, y_stride, dev->status));
  };
  if (dtype == CDGRAB_F32) return out_dtype == CDGRAB_F32 ? go(0.0f, 0.0f) : go(0.0f, __nv_bfloat16());
  return out_dtype == CDGRAB_F32 ? go(__nv_bfloat16(), 0.0f) : go(__nv_bfloat16(), __nv_bfloat16());
}

extern "C" long long cdgrab_embedding_workspace_bytes(int m, long long tokens, int cols, int vocab) {
  if (m < 1 || m > 65535 || tokens < 0 || cols < 1 || vocab < 1 || (tokens > 0 && m >= ((1ll << 31) + tokens - 1) / tokens)) return -1;
  return 16;
}

extern "C" int cdgrab_embedding_backward(int m, long long groups, long long length, int cols, int vocab, int token_bits,
                                         const void *tokens, long long token_stride, long long padding, float scale, int dtype,
                                         const void *dy, long long dy_stride, int grad_dtype, void *dtable, long long worker_stride,
                                         long long row_stride, int accumulate, void *workspace, long long workspace_bytes,
                                         void *stream) {
  if (groups < 0 || length < 0 || (length > 0 && groups >= ((1ll << 31) + length - 1) / length)) return CDGRAB_ERR_INVALID;
  const long long n = groups * length, need = cdgrab_embedding_workspace_bytes(m, n, cols, vocab);
  if (need < 0 || (token_bits != 32 && token_bits != 64) || !std::isfinite(scale) || !dtype_ok(dtype) || !dtype_ok(grad_dtype) ||
      (accumulate != 0 && accumulate != 1))
    return CDGRAB_ERR_INVALID;
  if (accumulate && n == 0) return CDGRAB_OK;
  if (!dtable || (vocab > 1 && row_stride < cols) || row_stride > (1ll << 31) ||
      (m > 1 && worker_stride < (vocab - 1) * row_stride + cols) || !cdg_aligned(dtable, size_of(grad_dtype)))
    return CDGRAB_ERR_INVALID;
  if (n > 0 && (!tokens || !dy || (m * groups > 1 && token_stride < length) || (m * n > 1 && dy_stride < cols) ||
                !cdg_aligned(tokens, token_bits / 8) || !cdg_aligned(dy, size_of(dtype))))
    return CDGRAB_ERR_INVALID;
  if (!workspace || workspace_bytes < need || !cdg_aligned(workspace, 16)) return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  const Tokens tok = {tokens, token_bits, token_stride, length, padding, vocab};
  cudaStream_t st = (cudaStream_t)stream;
  auto go = [&](auto t, auto g) {
    using T = decltype(t);
    using G = decltype(g);
    return cdg_launch_rc(cdg_ops_launch(gradient_kernel<T, G>, dim3(((unsigned)vocab + kWarps - 1) / kWarps, m), kThreads, 0, st, groups, cols,
                                        tok, scale, (const T *)dy, dy_stride, (G *)dtable, worker_stride, row_stride, accumulate,
                                        dev->status));
  };
  if (dtype == CDGRAB_F32) return grad_dtype == CDGRAB_F32 ? go(0.0f, 0.0f) : go(0.0f, __nv_bfloat16());
  return grad_dtype == CDGRAB_F32 ? go(__nv_bfloat16(), 0.0f) : go(__nv_bfloat16(), __nv_bfloat16());
}
