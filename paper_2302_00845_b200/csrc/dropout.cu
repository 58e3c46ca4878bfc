// Dropout from a counter-based generator, onto a residual stream or alone; the backward pass draws the same mask again.
//
//   y = residual + keep x / q,  keep_i = (bits_i >= T),  T = round(65536 p),  q = 1 - T / 65536,
// bits_i the i % 8-th 16 bits of Philox4x32-10(key = seed, counter = (i / 8, call, step)).
#include <cmath>

#include "philox.cuh"
#include "rows.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kBlocks = 2;         // blocks of eight elements to a thread

struct Draw {
  uint32_t key[10][2];         // of each round
  uint32_t call, step;
  const long long *step_dev;
  uint32_t limit;              // T 2^16
  float factor;                // 1 / q
};

// the four words of block b
__device__ __forceinline__ void draw_block(const Draw &d, uint32_t step, long long b, uint32_t (&c)[4]) {
  c[0] = (uint32_t)b;
  c[1] = (uint32_t)(b >> 32);
  c[2] = d.call;
  c[3] = step;
#pragma unroll
  for (int i = 0; i < 10; ++i) cdg_philox_round(c[0], c[1], c[2], c[3], d.key[i][0], d.key[i][1]);
}
// A half-word is compared where it stands at the top of a word: what lies below it cannot change the result against T 2^16.
__device__ __forceinline__ bool kept(const Draw &d, uint32_t word, int e) { return (e % 2 ? word : word << 16) >= d.limit; }

// A thread takes kBlocks blocks of eight elements, each one access of 16 or 32 bytes: their values are requested, then the generator
// runs while they are on their way.  Sixteen bits an element rather than a word: the ten rounds are 40 instructions, and at two
// bytes in and two out an element an SM has 22 issue slots for each.
// Blocks are numbered through rows of per_row blocks; FLAT: one row of n values, the last block perhaps cut short.
// x = NULL: all is dropped.
// (65,536 x 768 bf16: 36.6 us, 5.5 TB/s; one block to a thread 38.3, four 36.7.  Held to 48 registers, four spill.)
template <typename T, typename R, bool RES, bool FLAT>
__global__ void __launch_bounds__(kThreads) dropout_kernel(long long n, long long blocks, CdgDivisor per_row, const T *x, long long xs,
                                                           const R *res, long long rs, R *y, long long ys,
                                                           const __grid_constant__ Draw d) {
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const uint32_t step = d.step + (d.step_dev ? (uint32_t)*d.step_dev : 0u);
  const long long base = (long long)blockIdx.x * (kThreads * kBlocks);
  const long long first = FLAT ? 0 : base / per_row.d;
  const uint32_t off = FLAT ? threadIdx.x : (uint32_t)(base - first * per_row.d) + threadIdx.x;
  CdgVec<T, 8> vx[kBlocks];
  CdgVec<R, 8> vr[kBlocks];
  auto place = [&](int u, long long stride) {
    if (FLAT) return (base + threadIdx.x + u * kThreads) * 8;
    const uint32_t i = off + u * kThreads, q = cdg_divide(i, per_row);
    return (first + q) * stride + (i - q * per_row.d) * 8ll;
  };
#pragma unroll
  for (int u = 0; u < kBlocks; ++u) {
    const long long b = base + threadIdx.x + u * kThreads;
    const bool some = FLAT ? b * 8 + 8 <= n : b < blocks;
    vx[u].zero();
    vx[u].load_if(some && x, x + place(u, xs));
    if (RES) {
      vr[u].zero();
      vr[u].load_if(some, res + place(u, rs));
    }
  }
#pragma unroll
  for (int u = 0; u < kBlocks; ++u) {
    const long long b = base + threadIdx.x + u * kThreads;
    if (b >= blocks) break;
    uint32_t c[4];
    draw_block(d, step, b, c);
    if (!FLAT || b * 8 + 8 <= n) {
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = kept(d, c[e / 2], e) ? vx[u].get(e) : 0.0f;
        f[e] = RES ? fmaf(v, d.factor, vr[u].get(e)) : v * d.factor;
      }
      CdgVec<R, 8> o;
      o.set(f);
      o.store(y + place(u, ys));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const long long i = b * 8 + e;
        if (i >= n) break;
        const float v = x && kept(d, c[e / 2], e) ? cdg_ld(x + i) : 0.0f;
        y[i] = cdg_cast<R>(RES ? fmaf(v, d.factor, cdg_ld(res + i)) : v * d.factor);
      }
    }
  }
}

// rows that no wide access fits: a thread to a block, value by value
template <typename T, typename R>
__global__ void __launch_bounds__(kThreads) dropout_narrow_kernel(long long n, long long cols, const T *x, long long xs, const R *res,
                                                                  long long rs, R *y, long long ys, const __grid_constant__ Draw d) {
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const uint32_t step = d.step + (d.step_dev ? (uint32_t)*d.step_dev : 0u);
  const long long b = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (b * 8 >= n) return;
  uint32_t c[4];
  draw_block(d, step, b, c);
  long long r = b * 8 / cols, k = b * 8 - r * cols;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (b * 8 + e >= n) break;
    const float v = x && kept(d, c[e / 2], e) ? cdg_ld(x + r * xs + k) : 0.0f;
    y[r * ys + k] = cdg_cast<R>(fmaf(v, d.factor, res ? cdg_ld(res + r * rs + k) : 0.0f));
    if (++k == cols) { k = 0; ++r; }
  }
}

int dropout(long long rows, long long cols, int dtype, const void *x, long long xs, int out_dtype, const void *res, long long rs,
            void *y, long long ys, double p, unsigned long long seed, unsigned call, unsigned step, const long long *step_dev,
            void *stream) {
  if (rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 31) || rows * cols >= (1ll << 42) || !cdg_dtype_ok(dtype) || !cdg_dtype_ok(out_dtype) ||
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
  Draw d = {};
  for (int i = 0; i < 10; ++i) {
    d.key[i][0] = (uint32_t)seed + i * kPhiloxWeyl0;
    d.key[i][1] = (uint32_t)(seed >> 32) + i * kPhiloxWeyl1;
  }
  d.call = call;
  d.step = step;
  d.step_dev = step_dev;
  d.limit = none ? 0u : limit << 16;
  d.factor = none ? 0.0f : (float)(65536.0 / (65536.0 - limit));
  const long long n = rows * cols, blocks = (n + 7) / 8;
  const bool flat = rows == 1 || (xs == cols && ys == cols && (!res || rs == cols));
  const bool wide = flat ? cdg_widest(8, {{x, 0, e}, {res, 0, oe}, {y, 0, oe}}) == 8
                         : cdg_widest(cols, {{x, xs, e}, {res, rs, oe}, {y, ys, oe}}) == 8;
  const long long grid = wide ? (blocks + kBlocks * kThreads - 1) / (kBlocks * kThreads) : (blocks + kThreads - 1) / kThreads;
  if (none) x = nullptr;
  cudaStream_t st = (cudaStream_t)stream;
  return cdg_by_types(dtype, out_dtype, [&](auto t, auto r) {
    using T = decltype(t);
    using R = decltype(r);
    if (!wide)
      return cdg_launch_rc(cdg_ops_launch(dropout_narrow_kernel<T, R>, dim3((unsigned)grid), kThreads, 0, st, n, cols, (const T *)x, xs,
                                          (const R *)res, rs, (R *)y, ys, d));
    auto go = [&](auto *kernel) {
      return cdg_launch_rc(cdg_ops_launch(kernel, dim3((unsigned)grid), kThreads, 0, st, n, blocks, cdg_divisor(flat ? 1u : (uint32_t)(cols / 8)),
                                          (const T *)x, xs, (const R *)res, rs, (R *)y, ys, d));
    };
    if (res) return flat ? go(dropout_kernel<T, R, true, true>) : go(dropout_kernel<T, R, true, false>);
    return flat ? go(dropout_kernel<T, R, false, true>) : go(dropout_kernel<T, R, false, false>);
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
