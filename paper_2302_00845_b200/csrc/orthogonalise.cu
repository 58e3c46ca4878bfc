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
// VEC values to a load: 16 bytes where rows, stride and address allow it, else one
template <typename T, int VEC>
__global__ void __launch_bounds__(256) orth_sumsq(const T *g, long long gb, long long gs, int rows, int cols,
                                                  double *part) {
  struct __align__(sizeof(T) * VEC) Piece { T v[VEC]; };
  __shared__ double sm[8];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const T *p = g + blockIdx.y * gb;
  const int per = cols / VEC;
  const long long all = (long long)rows * per, step = (long long)gridDim.x * 256;
  double s = 0.0;       // squares in 64 bits: entries of 1e-18 and 1e18 are taken as they are
#pragma unroll 4
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
    const long long r = i / per;
    const Piece q = *reinterpret_cast<const Piece *>(p + r * gs + (i - r * per) * VEC);
#pragma unroll
    for (int e = 0; e < VEC; ++e) { const double v = cdg_ld(&q.v[e]); s = fma(v, v, s); }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) s += sm[w];
    part[blockIdx.y * kNormBlocks + blockIdx.x] = s;
  }
}

// x[m][ldx] = kScale G (or its transpose) / (norm + eps), a tile of 64 x 64 to a block
template <typename T, int VEC>
__global__ void __launch_bounds__(256) orth_start(const T *g, long long gb, long long gs, int rows, int cols, int tall,
                                                  const double *part, float eps, __half *x, int ldx, long long xb) {
  struct __align__(sizeof(T) * VEC) Piece { T v[VEC]; };
  struct __align__(2 * VEC) Half { __half v[VEC]; };
  __shared__ double sm[4];
  __shared__ __half tile[64][66];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  constexpr int per = 64 / VEC, lines = 256 / per;        // loads to a row of the tile, rows at a time
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, tx = threadIdx.x % per * VEC, ty = threadIdx.x / per;
  const T *p = g + blockIdx.z * gb;
  Piece q[64 / lines];
#pragma unroll
  for (int i = 0; i < 64 / lines; ++i)
    if (r0 + ty + i * lines < rows && c0 + tx < cols) q[i] = *reinterpret_cast<const Piece *>(p + (r0 + ty + i * lines) * gs + c0 + tx);
  if (threadIdx.x < kNormBlocks) {
    double t = part[blockIdx.z * kNormBlocks + threadIdx.x];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = t;
  }
  __syncthreads();
  const double norm = sqrt(sm[0] + sm[1] + sm[2] + sm[3]) + (double)eps;
  const float f = norm > 0.0 ? (float)fmin((double)kScale / norm, 3e38) : 0.0f;
  __half *out = x + blockIdx.z * xb;
#pragma unroll
  for (int i = 0; i < 64 / lines; ++i) {
    const int r = ty + i * lines;
    if (r0 + r >= rows || c0 + tx >= cols) continue;
    Half h;
#pragma unroll
    for (int e = 0; e < VEC; ++e) h.v[e] = __float2half_rn(f * cdg_ld(&q[i].v[e]));
    if (tall) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) tile[tx + e][r] = h.v[e];
    } else if (VEC == 1 || ldx % VEC == 0) {
      *reinterpret_cast<Half *>(out + (long long)(r0 + r) * ldx + c0 + tx) = h;
    }
  }
  if (!tall) return;
  __syncthreads();
  // rows of x are columns of G: pairs of halves, whole 128-byte lines
  for (int i = threadIdx.x; i < 64 * 32; i += 256) {
    const int r = i >> 5, c = (i & 31) * 2;
    if (c0 + r >= cols) continue;
    __half *to = out + (long long)(c0 + r) * ldx + r0 + c;
    if (r0 + c + 1 < rows) *reinterpret_cast<__half2 *>(to) = *reinterpret_cast<const __half2 *>(&tile[r][c]);
    else if (r0 + c < rows) *to = tile[r][c];
  }
}

// ---- the products ----------------------------------------------------------------------------
// Persistent CTAs, one to an SM, take tiles of C = A op(B), 128 rows by BN columns: warp 0 keeps a ring of
// shared-memory stages full (64 of K each), warp 1 issues the matrix instructions, warps 2 to 5 read the
// accumulator, of which there are two in tensor memory so that one tile's products run under the other's
// epilogue, and write it through shared memory in whole rows.
// BN = 256 where there are tiles enough: a 128 x 128 product reads its operands from shared memory at the
// full 128 bytes a cycle, one of 128 x 256 at three quarters of that.
// Where there are few tiles, the K loop is dealt out over a cluster and the fp32 sums joined through
// distributed shared memory in the order of the ranks.
constexpr int kM = 128, kK = 64, kThreads = 192;
enum Product { kGram, kPoly, kApply, kLast };   // A = X X^T; B = aI + bA + cAA; X = B X; the same into O

struct ProductArgs {
  int m, n, k, tiles;      // C is m x n; tiles of one matrix
  float alpha, beta, diag; // C = alpha acc + beta D + diag I
  const __half *D;         // kPoly: A
  void *C;
  int ldc;                 // kLast: row stride of O
  long long cb, db;        // batch strides
  int tall, vec;           // kLast: write the transpose; rows of O are 16-byte aligned
  int *status;
};

template <int P, int BN> struct Shape {
  static constexpr bool symmetric = P == kGram || P == kPoly;
  static constexpr uint32_t a_bytes = kM * kK * 2, stage = a_bytes + BN * kK * 2;
  static constexpr int ring = BN == 256 ? 4 : symmetric ? 5 : 6;
  // per epilogue warp: rows of 64 halves (both halves of the tile's columns where a tile of D is fetched
  // ahead), and a transposed piece of 64 rows of 32
  static constexpr int row_pitch = 72, col_pitch = 40;
  static constexpr uint32_t rows_bytes = 32 * row_pitch * 2, cols_bytes = 64 * col_pitch * 2;
  static constexpr uint32_t cols_at = P == kPoly ? 2 * rows_bytes : P == kGram ? rows_bytes : 0;      // (O is written one way or the other)
  static constexpr uint32_t warp_bytes = cols_at + cols_bytes;
  static constexpr uint32_t staging = ring * stage, bars = staging + 4 * warp_bytes;
  static constexpr size_t smem = bars + 256;
};
template <int P, int BN> struct Bars {
  TcQueue queue;
  uint64_t full[Shape<P, BN>::ring], empty[Shape<P, BN>::ring], acc_full[2], acc_empty[2];
  uint32_t tmem;
};

__device__ __forceinline__ uint32_t sum_at(int row, int piece) {        // fp32 [128][128], 16-byte pieces permuted by row
  return (uint32_t)(row * 512 + (((piece & ~7) | ((piece ^ row) & 7)) << 4));
}
template <int P>
__device__ __forceinline__ uint32_t finish(float x, float y, float dx, float dy, int i, int j, const ProductArgs &p) {
  x *= p.alpha;
  y *= p.alpha;
  if (P == kPoly) {
    x = fmaf(p.beta, dx, x) + (i == j ? p.diag : 0.0f);
    y = fmaf(p.beta, dy, y) + (i == j + 1 ? p.diag : 0.0f);
  }
  if (P == kLast) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&h);
  }
  const __half2 h = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t *>(&h);
}
// `rows` rows of 8 * pieces halves from shared memory (pitch in halves) to C at (r0, c0), a whole warp; the
// workspace's rows are padded to multiples of 8 values, so whole pieces are written there
__device__ __forceinline__ void put(const __half *from, int pitch, int rows, int pieces, __half *C, long long ldc, int r0, int c0,
                                    int nr, int nc, bool padded, bool vec) {
  const int lane = threadIdx.x & 31;
  if (vec) {
    for (int i = lane; i < rows * pieces; i += 32) {
      const int r = i / pieces, c = i % pieces * 8;
      if (r0 + r >= nr || c0 + c >= nc) continue;
      __half *to = C + (long long)(r0 + r) * ldc + c0 + c;
      if (padded || c0 + c + 8 <= nc) *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(from + r * pitch + c);
      else for (int e = 0; e < nc - c0 - c; ++e) to[e] = from[r * pitch + c + e];
    }
  } else {
    for (int i = lane; i < rows * pieces * 8; i += 32) {
      const int r = i / (pieces * 8), c = i % (pieces * 8);
      if (r0 + r < nr && c0 + c < nc) C[(long long)(r0 + r) * ldc + c0 + c] = from[r * pitch + c];
    }
  }
}

template <int P, int BN>
__global__ void __launch_bounds__(kThreads, 1) orth_product(const __grid_constant__ CUtensorMap ta,
                                                            const __grid_constant__ CUtensorMap tb, const ProductArgs p) {
  typedef Shape<P, BN> S;
  extern __shared__ __align__(1024) uint8_t base[];
  static_assert(sizeof(Bars<P, BN>) <= 256 && S::smem <= 232448, "");
  Bars<P, BN> &bar = *reinterpret_cast<Bars<P, BN> *>(base + S::bars);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t ring = smem_u32(base);
  const int ranks = (int)tc_cluster_size(), rank = (int)tc_cluster_rank();

  if (threadIdx.x == 0) {
    tc_queue_init(bar.queue, 6);
    for (int s = 0; s < S::ring; ++s) { mbar_init(smem_u32(&bar.full[s]), 1); mbar_init(smem_u32(&bar.empty[s]), 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&bar.acc_full[s]), 1); mbar_init(smem_u32(&bar.acc_empty[s]), 4); }
    mbar_init_fence();
  }
  if (warp == 1) tc_alloc(&bar.tmem, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t acc = bar.tmem;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const long long deadline = clock64() + kCdgWaitCycles;
  const int nk = ((p.k + kK - 1) / kK - rank + ranks - 1) / ranks;       // this CTA's steps of K: rank, rank + ranks, ...

  struct Tile { int i0, j0, z; };
  auto tile_of = [&](long long at) {
    const int z = (int)(at / p.tiles), t = (int)(at % p.tiles);
    int ti, tj;
    if (S::symmetric) {      // tiles (ti, tj), ti <= tj, counted column by column
      tj = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
      while ((tj + 1) * (tj + 2) / 2 <= t) ++tj;
      while (tj * (tj + 1) / 2 > t) --tj;
      ti = t - tj * (tj + 1) / 2;
    } else {
      const int nt = (p.m + kM - 1) / kM;
      ti = t % nt;
      tj = t / nt;
    }
    return Tile{ti * kM, tj * BN, z};
  };
  const long long first = blockIdx.x / ranks;      // a cluster takes one tile and asks for no more

  if (warp == 0) {
    if (tc_elect()) {
      bool ok = true;
      int n = 0, seq = 0;
      for (long long at = first; at >= 0 && ok; at = ranks > 1 ? -1 : tc_queue_next_one(bar.queue, seq++, deadline, ok)) {
        if (ranks == 1 && !(ok = tc_queue_ask(bar.queue, seq, deadline))) break;
        const Tile t = tile_of(at);
        for (int it = 0; it < nk; ++it, ++n) {
          if (!(ok = tc_wait_released(bar.empty, n, S::ring, deadline))) break;
          const uint32_t full = smem_u32(&bar.full[n % S::ring]), a = ring + n % S::ring * S::stage, b = a + S::a_bytes;
          const int k0 = (rank + it * ranks) * kK;
          mbar_expect_tx(full, S::stage);
          tma_load_3d(a, &ta, k0, t.i0, t.z, full);
          if (S::symmetric) {
            tma_load_3d(b, &tb, k0, t.j0, t.z, full);
          } else {           // panels of 64 columns, 64 rows of K
#pragma unroll
            for (int c = 0; c < BN / 64; ++c) tma_load_3d(b + c * kK * 128, &tb, t.j0 + c * 64, k0, t.z, full);
          }
        }
      }
      if (!ok) {
        atomicOr(p.status, CDG_ST_TIMEOUT);
        if (ranks == 1) tc_drain(bar.queue.full, seq + 1, 2);
        tc_drain(bar.full, n, S::ring);
      }
    }
  } else if (warp == 1) {
    constexpr uint32_t idesc = tc_idesc(false, kM, BN, false, !S::symmetric);
    bool ok = true;
    int n = 0, seq = 0;
    for (long long at = first; at >= 0 && ok; at = ranks > 1 ? -1 : tc_queue_next(bar.queue, seq++, deadline, ok)) {
      const uint32_t d = acc + (seq & 1) * BN;
      if (seq >= 2 && !(ok = tc_wait(&bar.acc_empty[seq & 1], tc_parity(seq - 2, 2), deadline))) break;
      for (int it = 0; it < nk; ++it, ++n) {
        if (!(ok = tc_wait(&bar.full[n % S::ring], tc_parity(n, S::ring), deadline))) break;
        tc_fence_after();
        const uint32_t a = ring + n % S::ring * S::stage, b = a + S::a_bytes;
        const uint64_t da = tc_desc_k(a), db = S::symmetric ? tc_desc_k(b) : tc_desc_mn(b, kK * 128);
        if (tc_elect()) {
#pragma unroll
          for (int kk = 0; kk < kK / 16; ++kk) tc_mma(d, da + kk * 2, db + kk * (S::symmetric ? 2 : 128), idesc, it > 0 || kk > 0);
          tc_commit(&bar.empty[n % S::ring]);
        }
        __syncwarp();
      }
      if (!ok) break;
      if (tc_elect()) tc_commit(&bar.acc_full[seq & 1]);
      __syncwarp();
    }
    if (!ok && lane == 0) atomicOr(p.status, CDG_ST_TIMEOUT);
  } else {
    const int w = warp & 3, r = w * 32 + lane;         // warp w of the four reads lanes 32 w ... of the accumulator
    __half *rows = reinterpret_cast<__half *>(base + S::staging + w * S::warp_bytes);
    __half *cols = rows + S::cols_at / 2;
    bool ok = true;
    int seq = 0;
    for (long long at = first; at >= 0 && ok; at = ranks > 1 ? -1 : tc_queue_next(bar.queue, seq++, deadline, ok)) {
      const Tile t = tile_of(at);
      __half *C = static_cast<__half *>(p.C) + t.z * p.cb;
      if (P == kPoly && ranks == 1) {      // the tile of A that is added, while the products run
        const __half *D = p.D + t.z * p.db;
#pragma unroll 4
        for (int i = lane; i < 32 * 16; i += 32) {
          const int rr = i >> 4, c = (i & 15) * 8;
          if (t.i0 + w * 32 + rr < p.m && t.j0 + c < p.n)
            *reinterpret_cast<uint4 *>(rows + ((c >> 6) * 32 + rr) * S::row_pitch + (c & 63)) =
                *reinterpret_cast<const uint4 *>(D + (long long)(t.i0 + w * 32 + rr) * p.ldc + t.j0 + c);
        }
        __syncwarp();
      }
      if (!(ok = tc_wait(&bar.acc_full[seq & 1], tc_parity(seq, 2), deadline))) break;
      tc_fence_after();
      const uint32_t d = acc + ((uint32_t)(w * 32) << 16) + (seq & 1) * BN;
      if (ranks > 1) {
        // this CTA's sums into the ring, which no copy fills any more
#pragma unroll
        for (int c0 = 0; c0 < kM; c0 += 32) {
          uint32_t v[32] = {};
          if (nk > 0) { tc_load32(d + c0, v); tc_wait_ld(); }
#pragma unroll
          for (int i = 0; i < 8; ++i)
            *reinterpret_cast<uint4 *>(base + sum_at(r, (c0 >> 2) + i)) = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        }
        break;
      }
      const bool mirror = S::symmetric && t.i0 != t.j0, turned = P == kLast && p.tall;
#pragma unroll 1
      for (int c0 = 0; c0 < BN; c0 += 64) {
        uint32_t v[2][32];
        tc_load32(d + c0, v[0]);
        tc_load32(d + c0 + 32, v[1]);
        tc_wait_ld();
        if (c0 + 64 == BN) {               // the accumulator is in registers: the tile after next may use it
          tc_fence_before();
          tc_warp_arrive(&bar.acc_empty[seq & 1]);
        }
        __half *mine = rows + (P == kPoly ? (c0 >> 6) * 32 * S::row_pitch : 0) + lane * S::row_pitch;
#pragma unroll
        for (int c = 0; c < 64; c += 8) {
          uint32_t o[4], dd[4] = {};
          if (P == kPoly) {
            const uint4 q = *reinterpret_cast<const uint4 *>(mine + c);
            dd[0] = q.x; dd[1] = q.y; dd[2] = q.z; dd[3] = q.w;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&dd[e]));
            o[e] = finish<P>(__uint_as_float(v[c >> 5][(c & 31) + 2 * e]), __uint_as_float(v[c >> 5][(c & 31) + 2 * e + 1]), f.x, f.y,
                             t.i0 + r, t.j0 + c0 + c + 2 * e, p);
            if (mirror || turned) {
              reinterpret_cast<uint16_t *>(cols)[(c + 2 * e) * S::col_pitch + lane] = (uint16_t)(o[e] & 0xffffu);
              reinterpret_cast<uint16_t *>(cols)[(c + 2 * e + 1) * S::col_pitch + lane] = (uint16_t)(o[e] >> 16);
            }
          }
          if (!turned) *reinterpret_cast<uint4 *>(mine + c) = make_uint4(o[0], o[1], o[2], o[3]);
        }
        __syncwarp();
        const int rr = t.i0 + w * 32, cc = t.j0 + c0;
        if (!turned) put(mine - lane * S::row_pitch, S::row_pitch, 32, 8, C, p.ldc, rr, cc, p.m, p.n, P != kLast, P != kLast || p.vec);
        if (mirror) put(cols, S::col_pitch, 64, 4, C, p.ldc, cc, rr, p.n, p.m, true, true);
        if (turned) put(cols, S::col_pitch, 64, 4, C, p.ldc, cc, rr, p.n, p.m, false, p.vec);
        __syncwarp();
      }
    }
    if (!ok && lane == 0) atomicOr(p.status, CDG_ST_TIMEOUT);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) { tc_fence_after(); tc_free(acc, 512); }
  if (ranks > 1) {
    tc_cluster_sync();
    // rank's share of the tile's rows: the cluster's sums added up, finished and written
    const Tile t = tile_of(first);
    const int share = kM / ranks, r0 = rank * share, e = threadIdx.x - 64;
    __half *C = static_cast<__half *>(p.C) + t.z * p.cb;
    __half *out = reinterpret_cast<__half *>(base + kM * 512);          // behind the sums: [share][136]
    if (e >= 0) {
      for (int i = e; i < share * 32; i += 128) {
        const int r = r0 + i / 32, piece = i % 32, c = piece * 4;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int k = 0; k < ranks; ++k) {
          const float4 u = tc_peer_load(ring + sum_at(r, piece), k);
          s.x += u.x; s.y += u.y; s.z += u.z; s.w += u.w;
        }
        float2 d0 = make_float2(0.0f, 0.0f), d1 = d0;
        if (P == kPoly && t.i0 + r < p.m && t.j0 + c < p.n) {
          const uint2 q = *reinterpret_cast<const uint2 *>(p.D + t.z * p.db + (long long)(t.i0 + r) * p.ldc + t.j0 + c);
          d0 = __half22float2(*reinterpret_cast<const __half2 *>(&q.x));
          d1 = __half22float2(*reinterpret_cast<const __half2 *>(&q.y));
        }
        *reinterpret_cast<uint2 *>(out + (i / 32) * 136 + c) =
            make_uint2(finish<P>(s.x, s.y, d0.x, d0.y, t.i0 + r, t.j0 + c, p), finish<P>(s.z, s.w, d1.x, d1.y, t.i0 + r, t.j0 + c + 2, p));
      }
      asm volatile("bar.sync 1, 128;" ::: "memory");
      const int w = e >> 5, per = share / 4;
      if (P == kLast && p.tall) {
        for (int i = e; i < kM * share; i += 128) {
          const int c = i / share, r = i % share;
          if (t.j0 + c < p.n && t.i0 + r0 + r < p.m) C[(long long)(t.j0 + c) * p.ldc + t.i0 + r0 + r] = out[r * 136 + c];
        }
      } else {
        put(out + w * per * 136, 136, per, 16, C, p.ldc, t.i0 + r0 + w * per, t.j0, p.m, p.n, P != kLast, P != kLast || p.vec);
      }
      if (S::symmetric && t.i0 != t.j0)
        for (int i = e; i < kM * (share / 8); i += 128) {
          const int c = i / (share / 8), r = i % (share / 8) * 8;
          if (t.j0 + c >= p.n || t.i0 + r0 + r >= p.m) continue;
          uint32_t q[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            q[k] = (uint32_t)__half_as_ushort(out[(r + 2 * k) * 136 + c]) | (uint32_t)__half_as_ushort(out[(r + 2 * k + 1) * 136 + c]) << 16;
          *reinterpret_cast<uint4 *>(C + (long long)(t.j0 + c) * p.ldc + t.i0 + r0 + r) = make_uint4(q[0], q[1], q[2], q[3]);
        }
    }
    tc_cluster_sync();           // no CTA leaves while another reads its sums
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

template <int P, int BN>
int launch(const CUtensorMap &ta, const CUtensorMap &tb, const ProductArgs &a, int batch, int cluster, cudaStream_t st) {
  static CdgPerDevice flags;
  if (!tc_raise_limit(flags, orth_product<P, BN>, Shape<P, BN>::smem)) return CDGRAB_ERR_CUDA;
  return tc_launch_cluster(orth_product<P, BN>, dim3((unsigned)(a.tiles * batch * cluster)), cluster, kThreads, Shape<P, BN>::smem, st, ta, tb, a);
}

template <int P>
int product(const CUtensorMap &ta, const CUtensorMap &tb, ProductArgs a, int batch, int sms, cudaStream_t st) {
  const int mt = (a.m + kM - 1) / kM, nt = (a.n + kM - 1) / kM, wide = (a.n + 255) / 256;
  if (P == kApply || P == kLast) {
    // tiles of 256 columns while they still give every SM one
    if ((long long)mt * wide * batch >= sms) {
      a.tiles = mt * wide;
      return launch<P, P == kApply || P == kLast ? 256 : 128>(ta, tb, a, batch, 1, st);
    }
    a.tiles = mt * nt;
  } else {
    a.tiles = mt * (mt + 1) / 2;
  }
  // few tiles: as many CTAs to each as fit the SMs and leave two steps of K (64 each) to a CTA
  int c = 1;
  while (c < 8 && (long long)a.tiles * batch * 2 * c <= sms && (a.k + kK - 1) / kK >= 4 * c) c *= 2;
  return launch<P, 128>(ta, tb, a, batch, c, st);
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
    if (!tc_encode(&tx[i], false, x[i], 3, dx, sx, kM) || !tc_encode(&tk[i], false, x[i], 3, dx, sx, kK)) return CDGRAB_ERR_CUDA;
  if (!tc_encode(&ta, false, A, 3, da, sa, kM) || !tc_encode(&tb, false, B, 3, da, sa, kM)) return CDGRAB_ERR_CUDA;

  const dim3 gt((cols + 63) / 64, (rows + 63) / 64, batch);
  const int e = dtype == CDGRAB_F32 ? 4 : 2;
  const bool wide = cdg_aligned(g, 16) && gs % (16 / e) == 0 && gb % (16 / e) == 0 && cols % (16 / e) == 0;
  int rc;
  auto begin = [&](auto *sumsq, auto *start, const auto *from) {
    const int r = cdg_launch_rc(cdg_ops_launch(sumsq, dim3(kNormBlocks, batch), 256, 0, st, from, gb, gs, rows, cols, part));
    return r != CDGRAB_OK ? r : cdg_launch_rc(cdg_ops_launch(start, gt, 256, 0, st, from, gb, gs, rows, cols, tall, part, eps, x[0], p.ldx, xb));
  };
  if (dtype == CDGRAB_F32)
    rc = wide ? begin(orth_sumsq<float, 4>, orth_start<float, 4>, (const float *)g) : begin(orth_sumsq<float, 1>, orth_start<float, 1>, (const float *)g);
  else
    rc = wide ? begin(orth_sumsq<__nv_bfloat16, 8>, orth_start<__nv_bfloat16, 8>, (const __nv_bfloat16 *)g)
              : begin(orth_sumsq<__nv_bfloat16, 1>, orth_start<__nv_bfloat16, 1>, (const __nv_bfloat16 *)g);
  const ProductArgs gram = {m, m, n, 0, 1.0f / (kScale * kScale), 0.0f, 0.0f, nullptr, A, p.lda, ab, 0, 0, 1, dev->status};
  const ProductArgs poly = {m, m, m, 0, coeffs[2], coeffs[1], coeffs[0], A, B, p.lda, ab, ab, 0, 1, dev->status};
  const ProductArgs last = {m, n, m, 0, 1.0f / kScale, 0.0f, 0.0f, nullptr, o, (int)os, ob, 0, tall,
                            cdg_aligned(o, 16) && os % 8 == 0 && ob % 8 == 0, dev->status};
  for (int i = 0; i < steps && rc == CDGRAB_OK; ++i) {
    const int at = i & 1;
    rc = product<kGram>(tx[at], tx[at], gram, batch, dev->sms, st);
    if (rc == CDGRAB_OK) rc = product<kPoly>(ta, ta, poly, batch, dev->sms, st);
    if (rc != CDGRAB_OK) break;
    if (i + 1 < steps) {
      const ProductArgs apply = {m, n, m, 0, 1.0f, 0.0f, 0.0f, nullptr, x[1 - at], p.ldx, xb, 0, 0, 1, dev->status};
      rc = product<kApply>(tb, tk[at], apply, batch, dev->sms, st);
    } else {
      rc = product<kLast>(tb, tk[at], last, batch, dev->sms, st);
    }
  }
  return rc;
}
