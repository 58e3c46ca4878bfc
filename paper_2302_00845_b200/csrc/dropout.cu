// Dropout from a counter-based generator, onto a residual stream or alone; the backward pass draws the same mask again.
//
//   y = residual + keep x / q,  keep_i = (bits_i >= T),  T = round(65536 p),  q = 1 - T / 65536,
// bits_i the i % 8-th 16 bits of Philox4x32-10(key = seed, counter = (i / 8, call, step)).
#include <cmath>

#include "philox.cuh"
#include "rows.cuh"

namespace {

constexpr int kThreads = 256;

struct Draw {
  uint32_t seed_lo, seed_hi, call, step;
  const long long *step_dev;
  uint32_t limit;      // T 2^16
  float factor;        // 1 / q
};

// A thread takes blocks of eight elements, kBlocks of them at a time: their values are requested, then the generator runs
// while they are on their way.  Sixteen bits an element rather than a word: ten rounds cost 60 to 70 instructions, and at two
// words of memory traffic an element, bf16 in and out, an SM has 22 issue slots for each.
// A half-word is compared where it stands at the top of a word: what lies below it cannot change the result against T 2^16.
// With T = 65536 there is no such number; x is not read at all then.
// WIDE: the eight values of a block are one access, 16 or 32 bytes; else one by one, in rows of any stride.
template <typename T, typename R, bool WIDE>
__global__ void __launch_bounds__(kThreads) dropout_kernel(long long n, long long cols, const T *x, long long xs, const R *res,
                                                           long long rs, R *y, long long ys, Draw d) {
  constexpr int kBlocks = 2;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const uint32_t step = d.step + (d.step_dev ? (uint32_t)*d.step_dev : 0u);
  const long long blocks = (n + 7) / 8;
  for (long long b0 = (long long)blockIdx.x * kThreads * kBlocks + threadIdx.x; b0 < blocks; b0 += (long long)gridDim.x * kThreads * kBlocks) {
    CdgVec<T, 8> vx[kBlocks];
    CdgVec<R, 8> vr[kBlocks];
    long long row[kBlocks], col[kBlocks];
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) {
      const long long at = (b0 + u * kThreads) * 8;
      row[u] = 0;
      col[u] = at;
      if (cols < n) {        // (what is contiguous throughout comes as one row)
        row[u] = n <= 0xffffffffll ? (uint32_t)at / (uint32_t)cols : at / cols;
        col[u] = at - row[u] * cols;
      }
      if (WIDE && at + 8 <= n) {
        if (x) vx[u].load(x + row[u] * xs + col[u]);
        else vx[u].zero();
        if (res) vr[u].load(res + row[u] * rs + col[u]);
        else vr[u].zero();
      }
    }
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) {
      const long long b = b0 + u * kThreads;
      if (b >= blocks) break;
      uint32_t c[4] = {(uint32_t)b, (uint32_t)(b >> 32), d.call, step};
      cdg_philox4x32_10(c[0], c[1], c[2], c[3], d.seed_lo, d.seed_hi);
      if (WIDE && b * 8 + 8 <= n) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool keep = (e % 2 ? c[e / 2] : c[e / 2] << 16) >= d.limit;
          f[e] = fmaf(keep ? vx[u].get(e) : 0.0f, d.factor, vr[u].get(e));
        }
        vr[u].set(f);
        vr[u].store(y + row[u] * ys + col[u]);
        continue;
      }
      long long r = row[u], k = col[u];
      for (int e = 0; e < 8 && b * 8 + e < n; ++e) {
        const uint32_t word = e < 2 ? c[0] : e < 4 ? c[1] : e < 6 ? c[2] : c[3];
        const bool keep = (e % 2 ? word : word << 16) >= d.limit;
        const float v = keep && x ? cdg_ld(x + r * xs + k) : 0.0f;
        y[r * ys + k] = cdg_cast<R>(fmaf(v, d.factor, res ? cdg_ld(res + r * rs + k) : 0.0f));
        if (++k == cols) { k = 0; ++r; }
      }
    }
  }
}

template <typename T, typename R, bool WIDE>
cudaError_t launch(long long n, long long cols, const void *x, long long xs, const void *res, long long rs, void *y, long long ys,
                   const Draw &d, cudaStream_t st) {
  const long long blocks = ((n + 7) / 8 + 2 * kThreads - 1) / (2 * kThreads);
  return cdg_ops_launch(dropout_kernel<T, R, WIDE>, dim3((unsigned)(blocks < (1ll << 30) ? blocks : 1ll << 30)), kThreads, 0, st, n, cols,
                        (const T *)x, xs, (const R *)res, rs, (R *)y, ys, d);
}

int dropout(long long rows, long long cols, int dtype, const void *x, long long xs, int out_dtype, const void *res, long long rs,
            void *y, long long ys, double p, unsigned long long seed, unsigned call, unsigned step, const long long *step_dev,
            void *stream) {
  if (rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 31) || !cdg_dtype_ok(dtype) || !cdg_dtype_ok(out_dtype) ||
      !(p >= 0.0 && p <= 1.0))
    return CDGRAB_ERR_INVALID;
  if (rows == 0 || cols == 0) return CDGRAB_OK;
  const int e = cdg_dtype_size(dtype), oe = cdg_dtype_size(out_dtype);
  if (!x || !y || xs < cols || ys < cols || (res && rs < cols) || !cdg_aligned(x, e) || !cdg_aligned(res, oe) ||
      !cdg_aligned(y, oe) || !cdg_aligned(step_dev, 8))
    return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  const uint32_t limit = (uint32_t)std::floor(p * 65536.0 + 0.5);
  const bool none = limit == 65536;
  const Draw d = {(uint32_t)seed, (uint32_t)(seed >> 32), call, step, step_dev, none ? 0u : limit << 16,
                  none ? 0.0f : (float)(65536.0 / (65536.0 - limit))};
  const long long n = rows * cols;
  if (xs == cols && ys == cols && (!res || rs == cols)) cols = n;          // one row
  // (the last elements of a single row go one by one)
  const bool wide = cdg_widest(cols == n ? 8 : cols, {{x, cols == n ? 0 : xs, e}, {res, cols == n ? 0 : rs, oe}, {y, cols == n ? 0 : ys, oe}}) == 8;
  if (none) x = nullptr;
  cudaStream_t st = (cudaStream_t)stream;
  return cdg_by_types(dtype, out_dtype, [&](auto t, auto r) {
    using T = decltype(t);
    using R = decltype(r);
    return cdg_launch_rc(wide ? launch<T, R, true>(n, cols, x, xs, res, rs, y, ys, d, st)
                              : launch<T, R, false>(n, cols, x, xs, res, rs, y, ys, d, st));
  });
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
