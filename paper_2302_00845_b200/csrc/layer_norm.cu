// Layer normalisation, forward and backward, with the weight's gradient reduced per worker.
//
// Forward:   mean = sum x / C,  var = sum (x - mean)^2 / C,  y = (x - mean) / sqrt(var + eps) * w + b.
// Backward:  n = (x - mean) rstd,  g = dy w,  dx = rstd (g - sum g / C - n (sum g n) / C),
//            dw = sum over a worker's rows of dy n,  db = the same of dy.
// Both are bound by memory where they are large: x is read and y written once forward; dy and x are read and dx
// written once backward, with the weight's sums in the same pass.  Statistics and sums are fp32; the
// variance is taken about the mean, a second pass over registers, not as a difference of two sums.
#include <initializer_list>

#include "operators.cuh"
#include "ptx.cuh"

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

// ---- rows of up to 8192 values: held in registers, one pass over memory ----------------------------
// A row belongs to a warp (up to 1024 columns) or to a block; a thread holds E = VEC x NV of its values,
// VEC adjacent ones to a load.  VEC is the widest that the row length and every pointer and stride
// allow: 16 bytes, two values, or one.  The next row is requested before the current one is reduced, so
// that loads are in flight during the shuffles.  (32 x 512 rows of 650 bf16, 4 bytes to a load: 13 us, 3.3 TB/s,
// and 15 with the host's call; 32 rows of 64: 14 us, all of it the host's call.)
template <int BYTES> struct Raw;
template <> struct Raw<16> { typedef uint4 type; };
template <> struct Raw<8> { typedef uint2 type; };
template <> struct Raw<4> { typedef uint32_t type; };
template <> struct Raw<2> { typedef uint16_t type; };

template <typename T, int VEC>
struct Vec {
  typedef typename Raw<sizeof(T) * VEC>::type raw;
  static __device__ __forceinline__ void open(const raw &r, float (&f)[VEC]) {
    const T *t = reinterpret_cast<const T *>(&r);
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[e] = cdg_ld(t + e);
  }
  static __device__ __forceinline__ raw close(const float (&f)[VEC]) {
    raw r;
    T *t = reinterpret_cast<T *>(&r);
#pragma unroll
    for (int e = 0; e < VEC; ++e) t[e] = cdg_cast<T>(f[e]);
    return r;
  }
};
// VEC floats of a parameter, or a constant where there is none
template <int VEC>
__device__ __forceinline__ void param(const float *p, int c, float other, float (&f)[VEC]) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[e] = other;
  } else if (VEC % 4 == 0) {
#pragma unroll
    for (int e = 0; e < VEC; e += 4) {
      const float4 v = *reinterpret_cast<const float4 *>(p + c + e);
      f[e] = v.x; f[(e + 1) % VEC] = v.y; f[(e + 2) % VEC] = v.z; f[(e + 3) % VEC] = v.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[e] = p[c + e];
  }
}

// sums of a and b over a row's threads
template <bool BLOCK>
__device__ __forceinline__ float2 row_sum(float a, float b, float2 *sm) {
  if (BLOCK) return block_sum(a, b, sm);
  return make_float2(cdg_warp_sum(a), cdg_warp_sum(b));
}

constexpr int kMaxWide = 512;             // threads to a row

template <typename T, int VEC, int NV, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? kMaxWide : kThreads)
ln_forward(long long rows, int cols, const T *x, long long xs, const float *__restrict__ w, const float *__restrict__ b,
           float eps, T *y, long long ys, float *mean_out, float *rstd_out) {
  typedef Vec<T, VEC> V;
  typedef typename V::raw raw;
  __shared__ float2 sm[BLOCK ? kMaxWide / 32 : 1];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int span = BLOCK ? blockDim.x : 32, l = BLOCK ? threadIdx.x : threadIdx.x & 31;
  const long long step = BLOCK ? gridDim.x : (long long)gridDim.x * kWarps;
  long long r = BLOCK ? blockIdx.x : (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int nv = cols / VEC;
  const float inv = 1.0f / (float)cols;
  raw next[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (r < rows && l + i * span < nv) next[i] = reinterpret_cast<const raw *>(x + r * xs)[l + i * span];
  for (; r < rows; r += step) {
    float v[NV][VEC], s = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (l + i * span < nv) {
        V::open(next[i], v[i]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s += v[i][e];
      }
    }
    if (r + step < rows) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (l + i * span < nv) next[i] = reinterpret_cast<const raw *>(x + (r + step) * xs)[l + i * span];
    }
    const float mean = row_sum<BLOCK>(s, 0.0f, sm).x * inv;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (l + i * span < nv) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) { v[i][e] -= mean; s = fmaf(v[i][e], v[i][e], s); }
      }
    const float rstd = 1.0f / sqrtf(row_sum<BLOCK>(s, 0.0f, sm).x * inv + eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = l + i * span;
      if (c < nv) {
        float fw[VEC], fb[VEC];
        param<VEC>(w, c * VEC, 1.0f, fw);
        param<VEC>(b, c * VEC, 0.0f, fb);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i][e] = fmaf(v[i][e] * rstd, fw[e], fb[e]);
        reinterpret_cast<raw *>(y + r * ys)[c] = V::close(v[i]);
      }
    }
    if (l == 0) {
      if (mean_out) mean_out[r] = mean;
      if (rstd_out) rstd_out[r] = rstd;
    }
  }
}

// A block takes a chunk of one worker's rows (blockIdx.y) and keeps its sums of dy n and dy in registers,
// a thread those of its own columns; at the chunk's end the warps of a block are added up in order and the
// sums go to part[worker][chunk][2][cols], or, where a worker has one chunk, to the gradients.
// The sums fill most of the registers (2 E of 128), so rows on their way are kept in shared memory: a ring
// of kAhead rows to a warp, filled by asynchronous copies.  A thread copies and reads only its own values,
// so the ring needs no barrier.  (Held in registers, one row ahead, the kernel spilled and moved
// 2.2 TB/s at 64 x 1024 x 768 bf16; now 63 us and 4.8 TB/s there, bound by issue slots, 51 % of them taken, and the 16
// warps an SM that the registers leave.  7 x 333 x 1025 fp32, a block to a row and one value to a load: 16.5 us out of L2,
// 20.8 out of DRAM, and 24 us for the call with its join.)
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src) {
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES < 4 ? 4 : BYTES) : "memory");
}
template <int E, int BYTES> struct Ring { static constexpr int ahead = E * BYTES <= 64 ? 3 : 2; };
// bytes of dynamic shared memory: the ring, or the warps' sums, which take its place
constexpr size_t backward_smem(int threads, int e, int elem, bool block) {
  const size_t ring = (size_t)threads * e * elem * 2 * (e * elem <= 64 ? 3 : 2), sums = block ? 0 : (size_t)threads * e * 8;
  return ring > sums ? ring : sums;
}

template <typename T, int VEC, int NV, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? kMaxWide : kThreads, BLOCK ? 1 : 2)
ln_backward(long long rows, long long per, int cols, const T *dy, long long dys, const T *x, long long xs,
            const float *__restrict__ w, const float *__restrict__ mean, const float *__restrict__ rstd, T *dx, long long dxs,
            float *part, void *dw, void *db, long long ws, int grad_bf16) {
  typedef Vec<T, VEC> V;
  typedef typename V::raw raw;
  constexpr int E = VEC * NV, kAhead = Ring<E, sizeof(T)>::ahead;
  constexpr bool ringed = sizeof(raw) >= 4;         // the copies move 4 bytes at least; 2-byte rows are read directly
  extern __shared__ __align__(16) uint8_t dyn[];
  __shared__ float2 sm[BLOCK ? kMaxWide / 32 : 1];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int span = BLOCK ? blockDim.x : 32, l = BLOCK ? threadIdx.x : threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int step = BLOCK ? 1 : kWarps, nv = cols / VEC;
  const float inv = 1.0f / (float)cols;
  const long long base = (long long)blockIdx.y * rows;
  const long long end = base + min(rows, (long long)(blockIdx.x + 1) * per);
  long long r = base + blockIdx.x * per + (BLOCK ? 0 : warp);
  // [stage][x, dy][NV][span] raw values of this warp (or block)
  raw *ring = reinterpret_cast<raw *>(dyn) + (BLOCK ? 0 : warp * kAhead * 2 * NV * 32) + l;
  auto request = [&](long long at, int stage) {
    if (at < end) {
      raw *to = ring + stage * 2 * NV * span;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (l + i * span < nv) {
          copy_async<sizeof(raw)>(smem_u32(to + i * span), reinterpret_cast<const raw *>(x + at * xs) + l + i * span);
          copy_async<sizeof(raw)>(smem_u32(to + (NV + i) * span), reinterpret_cast<const raw *>(dy + at * dys) + l + i * span);
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float2 sw[E / 2] = {}, sb[E / 2] = {};
  if (ringed) {
#pragma unroll
    for (int k = 0; k < kAhead - 1; ++k) request(r + k * step, k);
  }
  float mu = 0.0f, rs = 0.0f;
  if (r < end) { mu = mean[r]; rs = rstd[r]; }
  for (int stage = 0; r < end; r += step, stage = stage + 1 == kAhead ? 0 : stage + 1) {
    if (E > 24) asm volatile("" ::: "memory");       // the weight is read again for each row: it would not fit in registers
    if (ringed) {
      request(r + (kAhead - 1) * step, stage == 0 ? kAhead - 1 : stage - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
    }
    float mu_next = 0.0f, rs_next = 0.0f;
    if (r + step < end) { mu_next = mean[r + step]; rs_next = rstd[r + step]; }
    // past the row's end x, dy and w are 0, and with them every term.  Between the two passes x stays as it was
    // read and g = dy w in fp32, up to 24 values a thread; reading dy and w again cost half of the shared
    // memory's and L1's bandwidth
    raw cx[NV] = {};
    auto dy_of = [&](int i) {
      return ringed ? ring[(stage * 2 * NV + NV + i) * span] : reinterpret_cast<const raw *>(dy + r * dys)[l + i * span];
    };
    float2 g[E / 2], s1 = make_float2(0.0f, 0.0f), s2 = s1;
    const float2 off = make_float2(-mu, -mu), by = make_float2(rs, rs);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = l + i * span;
      raw cd = {};
      float fx[VEC], fd[VEC], fw[VEC] = {};
      if (c < nv) {
        cx[i] = ringed ? ring[(stage * 2 * NV + i) * span] : reinterpret_cast<const raw *>(x + r * xs)[c];
        cd = dy_of(i);
        param<VEC>(w, c * VEC, 1.0f, fw);
      }
      V::open(cx[i], fx);
      V::open(cd, fd);
#pragma unroll
      for (int e = 0; e < VEC; e += 2) {
        const int k = (i * VEC + e) / 2;
        if (VEC == 1 && i % 2 == 1) {                // the other half of the pair before
          const float n = (fx[0] - mu) * rs;
          sw[k].y = fmaf(fd[0], n, sw[k].y);
          sb[k].y += fd[0];
          g[k].y = fd[0] * fw[0];
          s1.y += g[k].y;
          s2.y = fmaf(g[k].y, n, s2.y);
        } else if (VEC == 1) {
          const float n = (fx[0] - mu) * rs;
          sw[k].x = fmaf(fd[0], n, sw[k].x);
          sb[k].x += fd[0];
          g[k].x = fd[0] * fw[0];
          s1.x += g[k].x;
          s2.x = fmaf(g[k].x, n, s2.x);
        } else {
          const int f = (e + 1) % VEC;
          const float2 n = mul2(add2(make_float2(fx[e], fx[f]), off), by), d = make_float2(fd[e], fd[f]);
          sw[k] = fma2(d, n, sw[k]);
          sb[k] = add2(sb[k], d);
          g[k] = mul2(d, make_float2(fw[e], fw[f]));
          s1 = add2(s1, g[k]);
          s2 = fma2(g[k], n, s2);
        }
      }
    }
    if (dx) {
      if (E > 24) asm volatile("" ::: "memory");
      const float2 t = row_sum<BLOCK>(s1.x + s1.y, s2.x + s2.y, sm);
      const float2 c1 = make_float2(-t.x * inv, -t.x * inv), c2 = make_float2(-t.y * inv, -t.y * inv);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = l + i * span;
        if (c < nv) {
          float fx[VEC], fd[VEC], fw[VEC];
          V::open(cx[i], fx);
          if (E > 24) {
            V::open(dy_of(i), fd);
            param<VEC>(w, c * VEC, 1.0f, fw);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              const int k = i * VEC + e;
              (k % 2 ? g[k / 2].y : g[k / 2].x) = fd[e] * fw[e];
            }
          }
#pragma unroll
          for (int e = 0; e < VEC; e += 2) {
            const int k = (i * VEC + e) / 2, f = (e + 1) % VEC;
            if (VEC == 1) {
              fx[0] = rs * ((i % 2 ? g[k].y : g[k].x) + c1.x + (fx[0] - mu) * rs * c2.x);
            } else {
              const float2 n = mul2(add2(make_float2(fx[e], fx[f]), off), by), d = mul2(by, fma2(n, c2, add2(g[k], c1)));
              fx[e] = d.x;
              fx[f] = d.y;
            }
          }
          reinterpret_cast<raw *>(dx + r * dxs)[c] = V::close(fx);
        }
        if (E > 24) asm volatile("" ::: "memory");
      }
    }
    mu = mu_next;
    rs = rs_next;
  }
  if (!dw && !db) return;
  float *mine = part ? part + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 2 * cols : nullptr;
  auto put = [&](int c, float a, float b) {
    if (mine) { mine[c] = a; mine[cols + c] = b; return; }
    const long long at = (long long)blockIdx.y * ws + c;
    if (grad_bf16) {
      if (dw) static_cast<__nv_bfloat16 *>(dw)[at] = __float2bfloat16_rn(a);
      if (db) static_cast<__nv_bfloat16 *>(db)[at] = __float2bfloat16_rn(b);
    } else {
      if (dw) static_cast<float *>(dw)[at] = a;
      if (db) static_cast<float *>(db)[at] = b;
    }
  };
  if (BLOCK) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (l + i * span < nv) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const int k = i * VEC + e;
          put((l + i * span) * VEC + e, k % 2 ? sw[k / 2].y : sw[k / 2].x, k % 2 ? sb[k / 2].y : sb[k / 2].x);
        }
      }
    return;
  }
  // [warp][dy n, dy][E][32]: written and read without bank conflicts
  float *sums = reinterpret_cast<float *>(dyn);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < E; ++k) {
    sums[(warp * 2 * E + k) * 32 + l] = k % 2 ? sw[k / 2].y : sw[k / 2].x;
    sums[(warp * 2 * E + E + k) * 32 + l] = k % 2 ? sb[k / 2].y : sb[k / 2].x;
  }
  __syncthreads();
  for (int k = warp; k < E; k += kWarps) {
    const int c = (l + k / VEC * 32) * VEC + k % VEC;
    if (c >= cols) continue;
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int o = 0; o < kWarps; ++o) { a += sums[(o * 2 * E + k) * 32 + l]; b += sums[(o * 2 * E + E + k) * 32 + l]; }
    put(c, a, b);
  }
}

// the chunks' sums of one worker (blockIdx.y) added up in order: 32 columns to a block, eight threads to a
// column, each every eighth chunk
template <typename G>
__global__ void __launch_bounds__(kThreads) ln_backward_join(int chunks, int cols, const float *__restrict__ part, G *dw, G *db,
                                                             long long ws) {
  __shared__ float sm[8][33];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const long long c = (long long)blockIdx.x * 32 + (threadIdx.x & 31), both = 2ll * cols;
  const int k0 = threadIdx.x >> 5;
  float s = 0.0f;
  if (c < both)
#pragma unroll 8
    for (int k = k0; k < chunks; k += 8) s += part[((long long)blockIdx.y * chunks + k) * both + c];
  sm[k0][threadIdx.x & 31] = s;
  __syncthreads();
  if (k0 == 0 && c < both) {
    for (int k = 1; k < 8; ++k) s += sm[k][threadIdx.x];
    G *out = c < cols ? dw : db;
    if (out) out[(long long)blockIdx.y * ws + (c < cols ? c : c - cols)] = cdg_cast<G>(s);
  }
}

// ---- longer rows ------------------------------------------------------------------------------------
// one block per row, three passes over it (columns counted without a sign: the last step may pass 2^31)
template <typename T>
__global__ void __launch_bounds__(kThreads) ln_forward_long(int cols, const T *__restrict__ x, long long xs,
                                                            const float *__restrict__ w, const float *__restrict__ b,
                                                            float eps, T *y, long long ys, float *mean_out,
                                                            float *rstd_out) {
  __shared__ float2 sm[kWarps];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const T *xr = x + (long long)blockIdx.x * xs;
  T *yr = y + (long long)blockIdx.x * ys;
  const unsigned n_cols = cols;
  const float inv = 1.0f / (float)cols;
  float s = 0.0f;
  for (unsigned c = threadIdx.x; c < n_cols; c += kThreads) s += cdg_ld(xr + c);
  const float mean = block_sum(s, 0.0f, sm).x * inv;
  s = 0.0f;
  for (unsigned c = threadIdx.x; c < n_cols; c += kThreads) { const float d = cdg_ld(xr + c) - mean; s += d * d; }
  const float rstd = 1.0f / sqrtf(block_sum(s, 0.0f, sm).x * inv + eps);
  for (unsigned c = threadIdx.x; c < n_cols; c += kThreads) {
    const float n = (cdg_ld(xr + c) - mean) * rstd;
    yr[c] = cdg_cast<T>(n * (w ? w[c] : 1.0f) + (b ? b[c] : 0.0f));
  }
  if (threadIdx.x == 0) {
    if (mean_out) mean_out[blockIdx.x] = mean;
    if (rstd_out) rstd_out[blockIdx.x] = rstd;
  }
}

// a worker's (blockIdx.z) sums of dy n and dy over a chunk (blockIdx.y) of its rows, one thread per column, before
// dx, which may overwrite dy or x; to part[worker][chunk][2][cols] where there are several chunks, else to the gradients
// (a worker's rows in one chain of additions: 20,000 equal gradients drifted by 1.7e-4 of their sum, and 4096 rows of 8193
// bf16 took 1602 us; in chunks 126 us, of which the two passes of dx are the larger part)
template <typename T, typename G>
__global__ void __launch_bounds__(kThreads) ln_backward_columns(long long rows, long long per, int cols, const T *__restrict__ dy,
                                                                long long dys, const T *__restrict__ x, long long xs,
                                                                const float *__restrict__ mean,
                                                                const float *__restrict__ rstd, float *part, G *dw, G *db,
                                                                long long ws) {
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const unsigned c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= (unsigned)cols) return;
  const long long r0 = (long long)blockIdx.z * rows, end = r0 + min(rows, (long long)(blockIdx.y + 1) * per);
  float sw = 0.0f, sb = 0.0f;
  for (long long r = r0 + blockIdx.y * per; r < end; ++r) {
    const float d = cdg_ld(dy + r * dys + c);
    sw += d * ((cdg_ld(x + r * xs + c) - mean[r]) * rstd[r]);
    sb += d;
  }
  if (part) {
    float *mine = part + ((long long)blockIdx.z * gridDim.y + blockIdx.y) * 2 * cols;
    mine[c] = sw;
    mine[(long long)cols + c] = sb;
    return;
  }
  if (dw) dw[(long long)blockIdx.z * ws + c] = cdg_cast<G>(sw);
  if (db) db[(long long)blockIdx.z * ws + c] = cdg_cast<G>(sb);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) ln_backward_long(int cols, const T *dy, long long dys, const T *x,
                                                             long long xs, const float *__restrict__ w,
                                                             const float *__restrict__ mean,
                                                             const float *__restrict__ rstd, T *dx, long long dxs) {
  __shared__ float2 sm[kWarps];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const long long r = blockIdx.x;
  const T *dyr = dy + r * dys, *xr = x + r * xs;
  T *dxr = dx + r * dxs;
  const unsigned n_cols = cols;
  const float mu = mean[r], rs = rstd[r], inv = 1.0f / (float)cols;
  float s1 = 0.0f, s2 = 0.0f;
  for (unsigned c = threadIdx.x; c < n_cols; c += kThreads) {
    const float g = cdg_ld(dyr + c) * (w ? w[c] : 1.0f);
    s1 += g;
    s2 += g * ((cdg_ld(xr + c) - mu) * rs);
  }
  const float2 t = block_sum(s1, s2, sm);
  for (unsigned c = threadIdx.x; c < n_cols; c += kThreads) {
    const float g = cdg_ld(dyr + c) * (w ? w[c] : 1.0f);
    const float n = (cdg_ld(xr + c) - mu) * rs;
    dxr[c] = cdg_cast<T>(rs * (g - t.x * inv - n * (t.y * inv)));
  }
}

inline bool dtype_ok(int t) { return t == CDGRAB_F32 || t == CDGRAB_BF16; }

// how a row is laid over threads
struct Layout {
  bool long_row;      // more than kMaxWide x 16 columns
  bool block;         // a block to a row
  int vec;            // 16-byte loads (0), two values (2) or one (1)
  int e;              // values to a thread: 8, 16, 24 or 32
  int threads;
};
// widest load that the columns, the strides (elements) and the addresses allow; parameters are read as floats
int widest(int elem, int cols, std::initializer_list<long long> strides, std::initializer_list<const void *> data,
           std::initializer_list<const void *> params) {
  for (int bytes : {16, 2 * elem}) {
    const int v = bytes / elem;
    bool ok = cols % v == 0;
    for (long long s : strides) ok = ok && s % v == 0;
    for (const void *p : data) ok = ok && cdg_aligned(p, bytes);
    if (v >= 4)
      for (const void *p : params) ok = ok && cdg_aligned(p, 16);
    if (ok) return bytes == 16 ? 0 : 2;
  }
  return 1;
}
Layout layout_of(int elem, int cols, int vec) {
  Layout l = {};
  l.vec = vec;
  l.long_row = cols > kMaxWide * 16;
  // up to 1024 columns a warp holds the row (32 values a lane) and needs no barrier; above, blocks of
  // ceil(cols / 16) threads
  if (l.long_row) return l;
  l.block = cols > 1024;
  l.e = l.block ? 16 : (cols + 255) / 256 * 8;
  l.threads = l.block ? ((cols + 15) / 16 + 31) / 32 * 32 : kThreads;
  return l;
}

template <typename T, int VEC, int E, bool BLOCK, typename F>
cudaError_t with_kernel(F &&f) { return f.template operator()<T, VEC, E / VEC, BLOCK>(); }
template <typename T, int VEC, typename F>
cudaError_t by_size(const Layout &l, F &&f) {
  if (l.block) return with_kernel<T, VEC, 16, true>(f);
  switch (l.e) {
    case 8: return with_kernel<T, VEC, 8, false>(f);
    case 16: return with_kernel<T, VEC, 16, false>(f);
    case 24: return with_kernel<T, VEC, 24, false>(f);
    default: return with_kernel<T, VEC, 32, false>(f);
  }
}
template <typename T, typename F>
cudaError_t by_layout(const Layout &l, F &&f) {
  return l.vec == 0 ? by_size<T, 16 / sizeof(T)>(l, f) : l.vec == 2 ? by_size<T, 2>(l, f) : by_size<T, 1>(l, f);
}

struct ForwardCall {
  long long rows; int cols; const void *x; long long xs; const float *w, *b; float eps; void *y; long long ys;
  float *mean, *rstd; Layout l; int sms; cudaStream_t st;
  template <typename T, int VEC, int NV, bool BLOCK> cudaError_t operator()() {
    const long long blocks = BLOCK ? rows : (rows + kWarps - 1) / kWarps;
    // rows beyond are looped over.  Eight blocks to an SM, one to two rounds of what is resident, even the loops out: at 4,
    // 6, 8 and 16, us: 16,384 rows of 650 bf16 14.0, 14.8, 13.0, 13.7; 65,536 of 768 40, 50, 41, 42; of 256 25, 18, 19, 18
    const long long most = (long long)sms * (BLOCK ? 2048 / l.threads : 8);
    return cdg_ops_launch(ln_forward<T, VEC, NV, BLOCK>, dim3((unsigned)(blocks < most ? blocks : most)), l.threads, 0, st, rows,
                          cols, (const T *)x, xs, w, b, eps, (T *)y, ys, mean, rstd);
  }
};

struct BackwardCall {
  int m; long long rows, per; int chunks, cols; const void *dy; long long dys; const void *x; long long xs;
  const float *w, *mean, *rstd; void *dx; long long dxs; float *part; void *dw, *db; long long ws; int grad_bf16;
  Layout l; int device; cudaStream_t st;
  template <typename T, int VEC, int NV, bool BLOCK> cudaError_t operator()() {
    static CdgPerDevice flags;
    const size_t smem = backward_smem(l.threads, VEC * NV, sizeof(T), BLOCK);
    const cudaError_t e = cdg_raise_smem_limit(flags, device, ln_backward<T, VEC, NV, BLOCK>,
                                               backward_smem(BLOCK ? kMaxWide : kThreads, VEC * NV, sizeof(T), BLOCK));
    if (e != cudaSuccess) return e;
    return cdg_ops_launch(ln_backward<T, VEC, NV, BLOCK>, dim3(chunks, m), l.threads, smem, st, rows, per,
                          cols, (const T *)dy, dys, (const T *)x, xs, w, mean, rstd, (T *)dx, dxs, part, dw, db, ws, grad_bf16);
  }
};

// Chunks to a worker: about two rounds of the blocks that are resident at once (two of eight warps to an SM,
// or, a block to a row, as many as 128 registers a thread allow), but at least a row to each warp, or two
// rows to a block of its own; one chunk where that leaves no more.
constexpr int kSms = 148;
int chunks_of(int m, long long rows, int cols) {
  const Layout l = layout_of(4, cols, 1);           // the threads depend on the columns alone
  if (l.long_row) {        // blocks of 256 columns, eight to an SM; at least 16 rows
    const long long blocks = ((long long)cols + kThreads - 1) / kThreads * m, most = 2 * 8 * kSms / blocks, fit = (rows + 15) / 16;
    const long long c = most < fit ? most : fit;
    return (int)(c < 1 ? 1 : c);
  }
  const long long resident = l.block ? 512 / l.threads : 2;
  const long long most = 2 * resident * kSms / m, fit = l.block ? (rows + 1) / 2 : (rows + kWarps - 1) / kWarps;
  const long long c = most < fit ? most : fit;
  return (int)(c < 1 ? 1 : c);
}

}  // namespace

extern "C" int cdgrab_layer_norm_forward(long long rows, int cols, int dtype, const void *x, long long xs,
                                         const float *w, const float *b, float eps, void *y, long long ys,
                                         float *mean, float *rstd, void *stream) {
  if (rows < 0 || rows >= (1ll << 31) || cols < 1 || !dtype_ok(dtype) || !(eps >= 0.0f)) return CDGRAB_ERR_INVALID;
  if (rows == 0) return CDGRAB_OK;
  if (!x || !y || xs < cols || ys < cols) return CDGRAB_ERR_INVALID;
  const int e = dtype == CDGRAB_F32 ? 4 : 2;
  if (!cdg_aligned(x, e) || !cdg_aligned(y, e) || !cdg_aligned(w, 4) || !cdg_aligned(b, 4) || !cdg_aligned(mean, 4) ||
      !cdg_aligned(rstd, 4))
    return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const Layout l = layout_of(e, cols, widest(e, cols, {xs, ys}, {x, y}, {w, b}));
  if (!l.long_row) {
    ForwardCall f = {rows, cols, x, xs, w, b, eps, y, ys, mean, rstd, l, dev->sms, st};
    return cdg_launch_rc(dtype == CDGRAB_F32 ? by_layout<float>(l, f) : by_layout<__nv_bfloat16>(l, f));
  }
  if (dtype == CDGRAB_F32)
    return cdg_launch_rc(cdg_ops_launch(ln_forward_long<float>, dim3((unsigned)rows), kThreads, 0, st, cols, (const float *)x, xs, w,
                                        b, eps, (float *)y, ys, mean, rstd));
  return cdg_launch_rc(cdg_ops_launch(ln_forward_long<__nv_bfloat16>, dim3((unsigned)rows), kThreads, 0, st, cols,
                                      (const __nv_bfloat16 *)x, xs, w, b, eps, (__nv_bfloat16 *)y, ys, mean, rstd));
}

extern "C" long long cdgrab_layer_norm_workspace_bytes(int m, long long rows, int cols) {
  if (m < 1 || m > 65535 || rows < 0 || cols < 1 || (rows > 0 && m >= (1ll << 31) / rows)) return -1;
  const int chunks = chunks_of(m, rows, cols);
  return chunks > 1 ? 8ll * m * chunks * cols : 16;
}

template <typename T, typename G>
static cudaError_t backward_long(const BackwardCall &c) {
  cudaError_t e = cudaSuccess;
  // (before dx, which may overwrite dy or x)
  if (c.dw || c.db)
    e = cdg_ops_launch(ln_backward_columns<T, G>, dim3(((unsigned)c.cols + kThreads - 1) / kThreads, c.chunks, c.m), kThreads, 0, c.st, c.rows,
                       c.per, c.cols, (const T *)c.dy, c.dys, (const T *)c.x, c.xs, c.mean, c.rstd, c.part, (G *)c.dw, (G *)c.db, c.ws);
  if (e == cudaSuccess && c.dx && c.rows)
    e = cdg_ops_launch(ln_backward_long<T>, dim3((unsigned)(c.m * c.rows)), kThreads, 0, c.st, c.cols, (const T *)c.dy, c.dys,
                       (const T *)c.x, c.xs, c.w, c.mean, c.rstd, (T *)c.dx, c.dxs);
  return e;
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
  const int e = dtype == CDGRAB_F32 ? 4 : 2, ge = grad_dtype == CDGRAB_F32 ? 4 : 2;
  if (!cdg_aligned(dy, e) || !cdg_aligned(x, e) || !cdg_aligned(dx, e) || !cdg_aligned(dw, ge) || !cdg_aligned(db, ge) ||
      !cdg_aligned(w, 4) || !cdg_aligned(mean, 4) || !cdg_aligned(rstd, 4))
    return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const Layout l = layout_of(e, cols, widest(e, cols, {xs, dys, dx ? dxs : 0}, {x, dy, dx}, {w}));
  const int chunks = chunks_of(m, rows, cols), gbf = grad_dtype == CDGRAB_BF16;
  BackwardCall c = {m, rows, (rows + chunks - 1) / chunks, chunks, cols, dy, dys, x, xs, w, mean, rstd, dx, dxs,
                    chunks > 1 ? (float *)workspace : nullptr, dw, db, ws, gbf, l, dev->index, st};
  int rc;
  if (l.long_row) {
    if (dtype == CDGRAB_F32) rc = cdg_launch_rc(gbf ? backward_long<float, __nv_bfloat16>(c) : backward_long<float, float>(c));
    else rc = cdg_launch_rc(gbf ? backward_long<__nv_bfloat16, __nv_bfloat16>(c) : backward_long<__nv_bfloat16, float>(c));
  } else {
    rc = cdg_launch_rc(dtype == CDGRAB_F32 ? by_layout<float>(l, c) : by_layout<__nv_bfloat16>(l, c));
  }
  if (rc == CDGRAB_OK && chunks > 1 && (dw || db)) {
    const dim3 grid((unsigned)((2ll * cols + 31) / 32), m);
    rc = cdg_launch_rc(gbf ? cdg_ops_launch(ln_backward_join<__nv_bfloat16>, grid, kThreads, 0, st, chunks, cols, c.part,
                                            (__nv_bfloat16 *)dw, (__nv_bfloat16 *)db, ws)
                           : cdg_ops_launch(ln_backward_join<float>, grid, kThreads, 0, st, chunks, cols, c.part, (float *)dw,
                                            (float *)db, ws));
  }
  return rc;
}
