// The orthogonalised update: Newton-Schulz products that drive a matrix's singular values to one.
//
//   X = G / (|G|_F + eps);  steps times:  A = X X^T,  X <- a X + (b A + c A A) X
// on the transposed matrix where G has more rows than columns (m <= n below).  Three products a step:
//
//   A = X X^T           symmetric: only the tiles on and above the diagonal, each written twice
//   B = a I + b A + c A A   symmetric likewise; the term a X is folded into the product that follows
//   X = B X             X's tiles as they lie are the MN-major operand: nothing is transposed
//
// Numerics.  Operands are fp16 (11 significant bits), sums fp32 in tensor memory.  X is held times
// kScale, so that entries down to 2.4e-7 stay normal numbers; nothing exceeds about 1.3 in X and 7 in
// B by the iteration's own bounds.  Each rounding is a choice: with bf16 operands the result is 1.1e-2
// off (2-norm, 768 x 768, half the energy in rank 16), with fp16 2.1e-3, of which 1.7e-3 is the bf16
// output's own rounding; a second fp16 term for X gained nothing more there.  Directions whose
// singular value is below about 2^-12 of the largest are dominated by that rounding, as they are by
// the rounding of G itself where G is bf16.
#include <cuda_fp16.h>
#include <math.h>

#include "tensor_core.cuh"

namespace {

constexpr float kScale = 256.0f;
constexpr int kNormBlocks = 128;

// ---- |G|_F ----------------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256) orth_sumsq(const T *g, long long gb, long long gs, int rows, int cols,
                                                  double *part) {
  __shared__ double sm[8];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const T *p = g + blockIdx.y * gb;
  double s = 0.0;       // squares in 64 bits: entries of 1e-18 and 1e18 are taken as they are
  for (int r = blockIdx.x; r < rows; r += gridDim.x)
    for (int c = threadIdx.x; c < cols; c += 256) { const double v = cdg_ld(p + r * gs + c); s += v * v; }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) s += sm[w];
    part[blockIdx.y * kNormBlocks + blockIdx.x] = s;
  }
}

// x[m][ldx] = kScale G (or its transpose) / (norm + eps), tiles of 64 x 64 through shared memory
template <typename T>
__global__ void __launch_bounds__(256) orth_start(const T *g, long long gb, long long gs, int rows, int cols, int tall,
                                                  const double *part, float eps, __half *x, int ldx, long long xb) {
  __shared__ double sm[4];
  __shared__ float tile[64][65];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  if (threadIdx.x < kNormBlocks) {
    double t = part[blockIdx.z * kNormBlocks + threadIdx.x];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = t;
  }
  __syncthreads();
  const double f = (double)kScale / (sqrt(sm[0] + sm[1] + sm[2] + sm[3]) + (double)eps);
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
  const T *p = g + blockIdx.z * gb;
  for (int i = ty; i < 64; i += 4)
    if (r0 + i < rows && c0 + tx < cols) tile[i][tx] = (float)(f * (double)cdg_ld(p + (r0 + i) * gs + c0 + tx));
  __syncthreads();
  __half *q = x + blockIdx.z * xb;
  for (int i = ty; i < 64; i += 4) {
    if (tall) {
      if (c0 + i < cols && r0 + tx < rows) q[(long long)(c0 + i) * ldx + r0 + tx] = __float2half_rn(tile[tx][i]);
    } else if (r0 + i < rows && c0 + tx < cols) {
      q[(long long)(r0 + i) * ldx + c0 + tx] = __float2half_rn(tile[i][tx]);
    }
  }
}

// ---- the products ----------------------------------------------------------------------------
// One CTA per 128 x 128 tile of C = A op(B): warp 0 keeps a ring of kStages shared-memory stages full
// (64 of K each), warp 1 issues the matrix instructions, then all four warps read the accumulator
// (128 columns of tensor memory) and write the tile through shared memory in whole rows.  A CTA takes
// 100 KB, so two share an SM and one's copies and epilogue run under the other's products.
constexpr int kTile = 128, kK = 64, kStages = 3;
constexpr uint32_t kOperandBytes = kTile * kK * 2, kStageBytes = 2 * kOperandBytes;
constexpr int kPitch = kTile + 8;        // halves per staged row: 16-byte accesses of eight rows hit all banks
constexpr size_t kProductSmem = kStages * kStageBytes + 1024;
static_assert(2 * kTile * kPitch * 2 <= kStages * kStageBytes, "the staged tiles reuse the ring");

enum Product { kGram, kPoly, kApply, kLast };   // A = X X^T; B = aI + bA + cAA; X = B X; the same into O

struct ProductArgs {
  int m, n, k;             // C is m x n
  float alpha, beta, diag; // C = alpha acc + beta D + diag I
  const __half *D;         // kPoly: A
  void *C;
  int ldc;                 // kLast: row stride of O
  long long cb, db;        // batch strides
  int tall, vec;           // kLast: write the transpose; rows of O are 16-byte aligned
  int *status;
};

template <int P>
__global__ void __launch_bounds__(128) orth_product(const __grid_constant__ CUtensorMap ta,
                                                    const __grid_constant__ CUtensorMap tb, const ProductArgs p) {
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t full[kStages], empty[kStages], done;
  __shared__ uint32_t tmem_slot;
  constexpr bool symmetric = P == kGram || P == kPoly;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, z = blockIdx.y;
  const uint32_t ring = (smem_u32(raw) + 1023u) & ~1023u;
  int ti, tj;
  if (symmetric) {         // tiles (ti, tj), ti <= tj, counted column by column
    tj = (int)((sqrtf(8.0f * (float)blockIdx.x + 1.0f) - 1.0f) * 0.5f);
    while ((tj + 1) * (tj + 2) / 2 <= (int)blockIdx.x) ++tj;
    while (tj * (tj + 1) / 2 > (int)blockIdx.x) --tj;
    ti = blockIdx.x - tj * (tj + 1) / 2;
  } else {
    const int nt = (p.m + kTile - 1) / kTile;
    ti = blockIdx.x % nt;
    tj = blockIdx.x / nt;
  }
  const int i0 = ti * kTile, j0 = tj * kTile, nk = (p.k + kK - 1) / kK;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { mbar_init(smem_u32(&full[s]), 1); mbar_init(smem_u32(&empty[s]), 1); }
    mbar_init(smem_u32(&done), 1);
    mbar_init_fence();
  }
  if (warp == 1) tc_alloc(&tmem_slot, kTile);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t acc = tmem_slot;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const long long deadline = clock64() + kCdgWaitCycles;

  if (warp == 0) {
    if (tc_elect()) {
      int it = 0;
      bool ok = true;
      for (; it < nk; ++it) {
        const int s = it % kStages;
        if (it >= kStages && !(ok = mbar_wait(smem_u32(&empty[s]), (it / kStages - 1) & 1, deadline))) break;
        const uint32_t bar = smem_u32(&full[s]), a = ring + s * kStageBytes, b = a + kOperandBytes;
        mbar_expect_tx(bar, kStageBytes);
        tma_load_3d(a, &ta, it * kK, i0, z, bar);
        if (P == kGram || P == kPoly) {
          tma_load_3d(b, &tb, it * kK, j0, z, bar);
        } else {          // two panels of 64 columns, 64 rows of K
          tma_load_3d(b, &tb, j0, it * kK, z, bar);
          tma_load_3d(b + kOperandBytes / 2, &tb, j0 + 64, it * kK, z, bar);
        }
      }
      if (!ok) {          // let the copies in flight land before the CTA gives up its shared memory
        atomicOr(p.status, CDG_ST_TIMEOUT);
        for (int i = max(0, it - kStages); i < it; ++i)
          mbar_wait(smem_u32(&full[i % kStages]), (i / kStages) & 1, clock64() + kCdgWaitCycles);
      }
    }
  } else if (warp == 1) {
    constexpr uint32_t idesc = tc_idesc(false, kTile, kTile, false, !symmetric);
    bool ok = true;
    for (int it = 0; it < nk; ++it) {
      const int s = it % kStages;
      if (!(ok = tc_wait(&full[s], (it / kStages) & 1, deadline))) break;
      tc_fence_after();
      const uint32_t a = ring + s * kStageBytes, b = a + kOperandBytes;
      const uint64_t da = tc_desc_k(a), db = symmetric ? tc_desc_k(b) : tc_desc_mn(b, kOperandBytes / 2);
      if (tc_elect()) {
#pragma unroll
        for (int kk = 0; kk < kK / 16; ++kk)
          tc_mma(acc, da + kk * 2, db + kk * (symmetric ? 2 : 128), idesc, it > 0 || kk > 0);
        tc_commit(&empty[s]);
      }
      __syncwarp();
    }
    if (!ok && lane == 0) atomicOr(p.status, CDG_ST_TIMEOUT);
    if (tc_elect()) tc_commit(&done);
    __syncwarp();
  }
  __syncwarp();

  // ---- epilogue: warp w holds rows 32 w ... of the tile
  const bool ok = mbar_wait(smem_u32(&done), 0, deadline + kCdgWaitCycles);
  if (!ok && lane == 0) atomicOr(p.status, CDG_ST_TIMEOUT);
  tc_fence_after();
  __syncthreads();            // no thread writes into the ring before all have seen the products end
  typedef __nv_bfloat16 bf16;
  __half *rows = reinterpret_cast<__half *>(raw + (ring - smem_u32(raw)));      // [128][kPitch]
  __half *cols = rows + kTile * kPitch;                                         // the transposed tile
  const int r = warp * 32 + lane;
  if (P == kPoly) {           // the tile of A that is added
    const __half *D = p.D + z * p.db;
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
      const int rr = warp * 32 + 2 * i + (lane >> 4), c = (lane & 15) * 8;
      if (i0 + rr < p.m && j0 + c < p.n)
        *reinterpret_cast<uint4 *>(rows + rr * kPitch + c) = *reinterpret_cast<const uint4 *>(D + (long long)(i0 + rr) * p.ldc + j0 + c);
    }
    __syncwarp();
  }
  const bool mirror = (symmetric && ti != tj) || (P == kLast && p.tall);
#pragma unroll
  for (int c0 = 0; c0 < kTile; c0 += 32) {
    uint32_t v[32];
    tc_load32(acc + ((uint32_t)(warp * 32) << 16) + c0, v);
    tc_wait_ld();
#pragma unroll
    for (int c = 0; c < 32; c += 8) {
      uint4 out;
      uint32_t *o = &out.x;
      if (P == kPoly) out = *reinterpret_cast<const uint4 *>(rows + r * kPitch + c0 + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float2 f = make_float2(__uint_as_float(v[c + 2 * e]) * p.alpha, __uint_as_float(v[c + 2 * e + 1]) * p.alpha);
        if (P == kPoly) {
          const float2 d = __half22float2(*reinterpret_cast<const __half2 *>(&o[e]));
          f.x += p.beta * d.x;
          f.y += p.beta * d.y;
          if (i0 + r == j0 + c0 + c + 2 * e) f.x += p.diag;
          if (i0 + r == j0 + c0 + c + 2 * e + 1) f.y += p.diag;
        }
        if (P == kLast) {
          const __nv_bfloat162 h = __float22bfloat162_rn(f);
          o[e] = *reinterpret_cast<const uint32_t *>(&h);
        } else {
          const __half2 h = __float22half2_rn(f);
          o[e] = *reinterpret_cast<const uint32_t *>(&h);
        }
        if (mirror) {
          reinterpret_cast<uint16_t *>(cols)[(c0 + c + 2 * e) * kPitch + r] = (uint16_t)(o[e] & 0xffffu);
          reinterpret_cast<uint16_t *>(cols)[(c0 + c + 2 * e + 1) * kPitch + r] = (uint16_t)(o[e] >> 16);
        }
      }
      *reinterpret_cast<uint4 *>(rows + r * kPitch + c0 + c) = out;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) { tc_fence_after(); tc_free(acc, kTile); }

  __half *C = static_cast<__half *>(p.C) + z * p.cb;
  if (P == kLast) {
    // O as the caller has it: rows of n (or of m, transposed) values
    const __half *src = p.tall ? cols : rows;
    const int ra = p.tall ? j0 : i0, ca = p.tall ? i0 : j0, nr = p.tall ? p.n : p.m, nc = p.tall ? p.m : p.n;
    if (p.vec) {
      for (int i = 0; i < 16; ++i) {
        const int rr = warp * 32 + 2 * i + (lane >> 4), c = (lane & 15) * 8;
        if (ra + rr >= nr) continue;
        __half *dst = C + (long long)(ra + rr) * p.ldc + ca + c;
        if (ca + c + 8 <= nc) {
          *reinterpret_cast<uint4 *>(dst) = *reinterpret_cast<const uint4 *>(src + rr * kPitch + c);
        } else {
          for (int e = 0; e < 8 && ca + c + e < nc; ++e) dst[e] = src[rr * kPitch + c + e];
        }
      }
    } else {
      for (int i = 0; i < 32; ++i) {
        const int rr = warp * 32 + i;
        if (ra + rr >= nr) break;
        for (int c = lane; c < kTile; c += 32)
          if (ca + c < nc) C[(long long)(ra + rr) * p.ldc + ca + c] = src[rr * kPitch + c];
      }
    }
    return;
  }
  // workspace rows are padded to multiples of 8 values: whole 16-byte pieces, the padding is never read
  for (int i = 0; i < 16; ++i) {
    const int rr = warp * 32 + 2 * i + (lane >> 4), c = (lane & 15) * 8;
    if (i0 + rr < p.m && j0 + c < p.n)
      *reinterpret_cast<uint4 *>(C + (long long)(i0 + rr) * p.ldc + j0 + c) = *reinterpret_cast<const uint4 *>(rows + rr * kPitch + c);
    if (symmetric && mirror && j0 + rr < p.n && i0 + c < p.m)
      *reinterpret_cast<uint4 *>(C + (long long)(j0 + rr) * p.ldc + i0 + c) = *reinterpret_cast<const uint4 *>(cols + rr * kPitch + c);
  }
}

inline long long up(long long v, long long to) { return (v + to - 1) / to * to; }

struct Plan {
  int m, n, ldx, lda;
  long long part, x0, x1, a, b, total;    // byte offsets in the workspace
};
Plan plan_of(long long batch, int rows, int cols) {
  Plan p;
  p.m = rows < cols ? rows : cols;
  p.n = rows < cols ? cols : rows;
  p.ldx = (int)up(p.n, 8);
  p.lda = (int)up(p.m, 8);
  const long long xb = up(2 * batch * p.m * p.ldx, 256), ab = up(2 * batch * p.m * p.lda, 256);
  p.part = 0;
  p.x0 = up(8 * batch * kNormBlocks, 256);
  p.x1 = p.x0 + xb;
  p.a = p.x1 + xb;
  p.b = p.a + ab;
  p.total = p.b + ab;
  return p;
}

template <int P>
int product(const CUtensorMap &ta, const CUtensorMap &tb, const ProductArgs &a, int batch, cudaStream_t st) {
  static CdgPerDevice flags;
  int dev = 0;
  cudaGetDevice(&dev);
  if (cdg_raise_smem_limit(flags, dev, orth_product<P>, kProductSmem) != cudaSuccess) return CDGRAB_ERR_CUDA;
  const int mt = (a.m + kTile - 1) / kTile, nt = (a.n + kTile - 1) / kTile;
  const int tiles = P == kGram || P == kPoly ? mt * (mt + 1) / 2 : mt * nt;
  return cdg_launch_rc(cdg_ops_launch(orth_product<P>, dim3(tiles, batch), 128, kProductSmem, st, ta, tb, a));
}

}  // namespace

extern "C" long long cdgrab_orthogonalise_workspace_bytes(int batch, int rows, int cols) {
  if (batch < 0 || batch > 65535 || rows < 0 || cols < 0 || rows > (1 << 20) || cols > (1 << 20)) return -1;
  return plan_of(batch, rows, cols).total + 256;
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
      os > 0x7fffffffll || (batch > 1 && (gb < 0 || ob < (long long)(rows - 1) * os + cols)))
    return CDGRAB_ERR_INVALID;
  if (!cdg_aligned(g, dtype == CDGRAB_F32 ? 4 : 2) || !cdg_aligned(o, 2)) return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const Plan p = plan_of(batch, rows, cols);
  const int tall = rows > cols, m = p.m, n = p.n;
  char *w = (char *)up((long long)(uintptr_t)workspace, 256);
  double *part = (double *)(w + p.part);
  __half *x[2] = {(__half *)(w + p.x0), (__half *)(w + p.x1)}, *A = (__half *)(w + p.a), *B = (__half *)(w + p.b);
  const long long xb = (long long)m * p.ldx, ab = (long long)m * p.lda;

  // X as 128-row boxes of 64 columns (operand of A) and as 64-row boxes (operand of B X); A and B
  CUtensorMap tx[2], tk[2], ta, tb;
  const long long dx[3] = {n, m, batch}, sx[3] = {1, p.ldx, xb}, da[3] = {m, m, batch}, sa[3] = {1, p.lda, ab};
  for (int i = 0; i < 2; ++i)
    if (!tc_encode(&tx[i], false, x[i], 3, dx, sx, kTile) || !tc_encode(&tk[i], false, x[i], 3, dx, sx, kK)) return CDGRAB_ERR_CUDA;
  if (!tc_encode(&ta, false, A, 3, da, sa, kTile) || !tc_encode(&tb, false, B, 3, da, sa, kTile)) return CDGRAB_ERR_CUDA;

  const dim3 gt((cols + 63) / 64, (rows + 63) / 64, batch);
  int rc;
  if (dtype == CDGRAB_F32) {
    rc = cdg_launch_rc(cdg_ops_launch(orth_sumsq<float>, dim3(kNormBlocks, batch), 256, 0, st, (const float *)g, gb, gs, rows, cols, part));
    if (rc == CDGRAB_OK)
      rc = cdg_launch_rc(cdg_ops_launch(orth_start<float>, gt, 256, 0, st, (const float *)g, gb, gs, rows, cols, tall, part, eps, x[0], p.ldx, xb));
  } else {
    rc = cdg_launch_rc(cdg_ops_launch(orth_sumsq<__nv_bfloat16>, dim3(kNormBlocks, batch), 256, 0, st, (const __nv_bfloat16 *)g, gb, gs, rows, cols, part));
    if (rc == CDGRAB_OK)
      rc = cdg_launch_rc(cdg_ops_launch(orth_start<__nv_bfloat16>, gt, 256, 0, st, (const __nv_bfloat16 *)g, gb, gs, rows, cols, tall, part, eps, x[0], p.ldx, xb));
  }
  const ProductArgs gram = {m, m, n, 1.0f / (kScale * kScale), 0.0f, 0.0f, nullptr, A, p.lda, ab, 0, 0, 1, dev->status};
  const ProductArgs poly = {m, m, m, coeffs[2], coeffs[1], coeffs[0], A, B, p.lda, ab, ab, 0, 1, dev->status};
  const ProductArgs last = {m, n, m, 1.0f / kScale, 0.0f, 0.0f, nullptr, o, (int)os, ob, 0, tall,
                            cdg_aligned(o, 16) && os % 8 == 0 && ob % 8 == 0, dev->status};
  for (int i = 0; i < steps && rc == CDGRAB_OK; ++i) {
    const int at = i & 1;
    rc = product<kGram>(tx[at], tx[at], gram, batch, st);
    if (rc == CDGRAB_OK) rc = product<kPoly>(ta, ta, poly, batch, st);
    if (rc != CDGRAB_OK) break;
    if (i + 1 < steps) {
      const ProductArgs apply = {m, n, m, 1.0f, 0.0f, 0.0f, nullptr, x[1 - at], p.ldx, xb, 0, 0, 1, dev->status};
      rc = product<kApply>(tb, tk[at], apply, batch, st);
    } else {
      rc = product<kLast>(tb, tk[at], last, batch, st);
    }
  }
  return rc;
}
