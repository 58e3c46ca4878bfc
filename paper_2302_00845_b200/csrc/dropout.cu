// Dropout from a counter-based generator, onto a residual stream or alone; the backward pass draws the same mask again.
//
//   y = residual + keep x / q,  keep_i = (bits_i >= T),  T = round(65536 p),  q = 1 - T / 65536,
// bits_i the i % 8-th 16 bits of Philox4x32-10(key = seed, counter = (i / 8, call, step)).
#include <cmath>

#include "operators.cuh"
#include "philox.cuh"

namespace {

constexpr int kThreads = 256;

struct Draw {
  uint32_t seed_lo, seed_hi, call, step;
  const long long *step_dev;
  uint32_t limit;      // T
  float factor;        // 1 / q, 0 where everything is dropped
};

// bit e of the result: element e of the block stays
__device__ __forceinline__ uint32_t keep_bits(const Draw &d, uint32_t step, long long block) {
  uint32_t c[4] = {(uint32_t)block, (uint32_t)(block >> 32), d.call, step};
  cdg_philox4x32_10(c[0], c[1], c[2], c[3], d.seed_lo, d.seed_hi);
  uint32_t k = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) k |= ((c[e / 2] >> (e % 2 * 16) & 0xffffu) >= d.limit ? 1u : 0u) << e;
  return k;
}

template <typename T, typename R>
__global__ void __launch_bounds__(kThreads) dropout_kernel(long long n, long long cols, const T *x, long long xs, const R *res,
                                                           long long rs, R *y, long long ys, Draw d) {
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const uint32_t step = d.step + (d.step_dev ? (uint32_t)*d.step_dev : 0u);
  for (long long b = (long long)blockIdx.x * kThreads + threadIdx.x; b * 8 < n; b += (long long)gridDim.x * kThreads) {
    const uint32_t keep = keep_bits(d, step, b);
    for (int e = 0; e < 8 && b * 8 + e < n; ++e) {
      const long long r = (b * 8 + e) / cols, c = (b * 8 + e) - r * cols;
      float v = keep >> e & 1 ? cdg_ld(x + r * xs + c) * d.factor : 0.0f;
      if (res) v += cdg_ld(res + r * rs + c);
      y[r * ys + c] = cdg_cast<R>(v);
    }
  }
}

inline bool dtype_ok(int t) { return t == CDGRAB_F32 || t == CDGRAB_BF16; }

template <typename T, typename R>
cudaError_t launch(long long n, long long cols, const void *x, long long xs, const void *res, long long rs, void *y, long long ys,
                   const Draw &d, int sms, cudaStream_t st) {
  const long long blocks = ((n + 7) / 8 + kThreads - 1) / kThreads, most = (long long)sms * 8;
  return cdg_ops_launch(dropout_kernel<T, R>, dim3((unsigned)(blocks < most ? blocks : most)), kThreads, 0, st, n, cols, (const T *)x,
                        xs, (const R *)res, rs, (R *)y, ys, d);
}

int dropout(long long rows, long long cols, int dtype, const void *x, long long xs, int out_dtype, const void *res, long long rs,
            void *y, long long ys, double p, unsigned long long seed, unsigned call, unsigned step, const long long *step_dev,
            void *stream) {
  if (rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 31) || !dtype_ok(dtype) || !dtype_ok(out_dtype) ||
      !(p >= 0.0 && p <= 1.0))
    return CDGRAB_ERR_INVALID;
  if (rows == 0 || cols == 0) return CDGRAB_OK;
  const int e = dtype == CDGRAB_F32 ? 4 : 2, oe = out_dtype == CDGRAB_F32 ? 4 : 2;
  if (!x || !y || xs < cols || ys < cols || (res && rs < cols) || !cdg_aligned(x, e) || !cdg_aligned(res, oe) ||
      !cdg_aligned(y, oe) || !cdg_aligned(step_dev, 8))
    return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  const uint32_t limit = (uint32_t)std::floor(p * 65536.0 + 0.5);
  const Draw d = {(uint32_t)seed, (uint32_t)(seed >> 32), call, step, step_dev, limit,
                  limit < 65536 ? (float)(65536.0 / (65536.0 - limit)) : 0.0f};
  const long long n = rows * cols;
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == CDGRAB_F32)
    return cdg_launch_rc(out_dtype == CDGRAB_F32 ? launch<float, float>(n, cols, x, xs, res, rs, y, ys, d, dev->sms, st)
                                                 : launch<float, __nv_bfloat16>(n, cols, x, xs, res, rs, y, ys, d, dev->sms, st));
  return cdg_launch_rc(out_dtype == CDGRAB_F32 ? launch<__nv_bfloat16, float>(n, cols, x, xs, res, rs, y, ys, d, dev->sms, st)
                                               : launch<__nv_bfloat16, __nv_bfloat16>(n, cols, x, xs, res, rs, y, ys, d, dev->sms, st));
}

}  // namespace

extern "C" int cdgrab_dropout_forward(long long rows, long long cols, int dtype, const void *x, long long xs, int out_dtype,
                                      const void *res, long long rs, void *y, long long ys, double p, unsigned long long seed,
                                      unsigned call, unsigned step, const long long *step_dev, void *stream) {
  return dropout(rows, cols, dtype, x, xs, out_dtype, res, rs, y, ys, p, seed, call, step, step_dev, stream);
}

extern "C" int cdgrab_dropout_backward(long long rows, long long cols, int dtype, const void *dy, long long dys, int out_dtype,
                                       void *dx, long long dxs, double p, unsigned long long seed, unsigned call, unsigned step,
                                       const long long *step_dev, void *stream) {
  return dropout(rows, cols, dtype, dy, dys, out_dtype, nullptr, 0, dx, dxs, p, seed, call, step, step_dev, stream);
}
