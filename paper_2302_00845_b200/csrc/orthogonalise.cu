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
// kScale, so that entries down to 2.4e-7 stay normal numbers; with the usual coefficients (3.4445, -4.7750, 2.0315)
// nothing exceeds about 1.3 in X and 4 in B, and others are refused where X, A or B might leave the
// type's range (in_range).  Each rounding is a choice: with bf16 operands the result is 1.1e-2
// off (2-norm, 768 x 768, half the energy in rank 16), with fp16 2.1e-3, of which 1.7e-3 is the bf16
// output's own rounding; a second fp16 term for X gained nothing more there.  Directions whose
// singular value is below about 2^-12 of the largest are dominated by that rounding, as they are by
// the rounding of G itself where G is bf16.
#include <cuda_fp16.h>
#include <math.h>

#include <atomic>

#include "tensor_core.cuh"

namespace {

constexpr float kScale = 256.0f;
constexpr int kNormBlocks = 128;

// ---- |G|_F ----------------------------------------------------------------------------------
// VEC values to a load: 16 bytes where rows, stride and address allow it, else one
template <typename T, int VEC>
__global__ void __launch_bounds__(256) orth_sumsq(const T *g, long long gb, long long gs, int rows, int cols,
                                                  double *part, unsigned *arrived) {
  struct __align__(sizeof(T) * VEC) Piece { T v[VEC]; };
  __shared__ double sm[8];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 2) arrived[threadIdx.x] = 0;       // the counters of orth_steps
  const T *p = g + blockIdx.y * gb;
  const int per = cols / VEC;
  const long long all = (long long)rows * per, step = (long long)gridDim.x * 256;
  double s = 0.0;       // squares in 64 bits: entries of 1e-18 and 1e18 are taken as they are
#pragma unroll 4
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
    const long long r = all < (1ll << 31) ? (long long)((unsigned)i / (unsigned)per) : i / per;      // (64-bit division is slow)
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
    } else {                 // (whole pieces: ldx is a multiple of 8)
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

// ---- the steps ---------------------------------------------------------------------------------
// One cooperative launch runs all steps: 3 x steps products with a barrier of the whole grid between them
// (17 launches took 164 us for one 650 x 2600 matrix, ten microseconds each whatever they did; at present 150 us in
// all there, mostly the latency of 15 dependent products, and 412 us, 660 TFLOP/s, for twelve of 2304 x 768: call after
// call, under the power cap, 17 and 28 us for the norm and the cast and 357 for the steps, which take 316 alone).  Persistent
// CTAs, one to an SM, take tiles of C = A op(B), 128 rows by 128 or BN columns: warp 0 keeps a ring of
// shared-memory stages full (64 of K each), warp 1 issues the matrix instructions, warps 2 to 5 read the
// accumulator, of which there are two in tensor memory so that one tile's products run under the other's
// epilogue, and write it through shared memory in whole rows.
//   BN = 256    for X = B X where there are tiles enough: what bounds large matrices is the operands' way
//               from L2 (11 TB/s), and the wider tile reads a quarter less of them
//   RANKS > 1   few tiles: CTAs form clusters, whose ranks share the K loop of a tile of A or B and join
//               their fp32 sums through distributed shared memory in the order of the ranks
constexpr int kM = 128, kK = 64, kThreads = 192;
enum Product { kGram, kPoly, kApply, kLast };   // A = X X^T; B = aI + bA + cAA; X = B X; the same into O

struct StepArgs {
  int m, n, batch, steps, ldx, lda, tall, vec;   // C is m x m, or m x n; vec: rows of O are 16-byte aligned
  float a, b, c;
  __half *x[2], *A, *B;
  void *o;
  long long xb, ab, ob, os;
  unsigned *arrived;         // [2] CTAs past each product of a part of the batch, counted on
  long long wait;            // how long the copies may wait for the grid or a stage, in clock cycles; what waits for them, twice and three times that
  int *status;
};
// X as rows of K and as panels of N, A and B; the same written in pieces of 32 x 32
struct StepMaps { CUtensorMap rows[2], panels[2], A, B, to_x[2], to_A, to_B; };

template <int BN, int RANKS> struct Shape {
  static constexpr uint32_t a_bytes = kM * kK * 2, stage = a_bytes + BN * kK * 2;
  static constexpr int ring = 4;
  // per epilogue warp two buffers of 32 x 32 halves and their transpose, swizzled as the copies read them (or,
  // written out by the warp itself, rows with these pitches)
  static constexpr uint32_t warp_bytes = 8192;
  static constexpr uint32_t sums = ring * stage, staging = sums + (RANKS > 1 ? kM * kM * 4 : 0), bars = staging + 4 * warp_bytes;
  static constexpr size_t smem = bars + 256;
};
template <int BN, int RANKS> struct Bars {
  uint64_t full[Shape<BN, RANKS>::ring], empty[Shape<BN, RANKS>::ring], acc_full[2], acc_empty[2], joined, read, finished;
  uint32_t tmem;
};

__device__ __forceinline__ uint32_t sum_at(int row, int piece) {        // fp32 [128][128], 16-byte pieces permuted by row
  return (uint32_t)(row * 512 + (((piece & ~7) | ((piece ^ row) & 7)) << 4));
}
// two values of a product as they are stored; d: the two of A that kPoly adds
template <int KIND>
__device__ __forceinline__ uint32_t finish(const StepArgs &p, float x, float y, uint32_t d, int i, int j) {
  if (KIND == kGram) { x *= 1.0f / (kScale * kScale); y *= 1.0f / (kScale * kScale); }
  if (KIND == kPoly) {
    const float2 q = __half22float2(*reinterpret_cast<const __half2 *>(&d));
    x = fmaf(p.b, q.x, x * p.c) + (i == j ? p.a : 0.0f);
    y = fmaf(p.b, q.y, y * p.c) + (i == j + 1 ? p.a : 0.0f);
  }
  if (KIND == kLast) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x * (1.0f / kScale), y * (1.0f / kScale));
    return *reinterpret_cast<const uint32_t *>(&h);
  }
  const __half2 h = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t *>(&h);
}
// O as the caller has it: nr x nc values, rows ld apart, on 16-byte boundaries where vec is set
struct Out { __half *p; long long ld; int nr, nc; bool vec; };
// ROWS rows of 8 * PIECES halves from shared memory (pitch in halves) to (r0, c0), a whole warp
template <int ROWS, int PIECES>
__device__ __forceinline__ void put(const __half *from, int pitch, const Out &o, int r0, int c0) {
  const int lane = threadIdx.x & 31;
  if (o.vec) {
#pragma unroll
    for (int i = 0; i < ROWS * PIECES / 32; ++i) {
      const int r = (i * 32 + lane) / PIECES, c = (i * 32 + lane) % PIECES * 8;
      if (r0 + r >= o.nr || c0 + c >= o.nc) continue;
      __half *to = o.p + (long long)(r0 + r) * o.ld + c0 + c;
      if (c0 + c + 8 <= o.nc) *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(from + r * pitch + c);
      else for (int e = 0; e < o.nc - c0 - c; ++e) to[e] = from[r * pitch + c + e];
    }
  } else {
    for (int i = lane; i < ROWS * PIECES * 8; i += 32) {
      const int r = i / (PIECES * 8), c = i % (PIECES * 8);
      if (r0 + r < o.nr && c0 + c < o.nc) o.p[(long long)(r0 + r) * o.ld + c0 + c] = from[r * pitch + c];
    }
  }
}

__device__ __forceinline__ bool wait_count(const unsigned *count, unsigned want, long long deadline) {
  unsigned got;
  while (true) {
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(got) : "l"(count) : "memory");
    if (got >= want) return true;
    if (clock64() > deadline) return false;
  }
}
// barrier of the four epilogue warps, and whether all of them are well: they go on, or leave, together
__device__ __forceinline__ bool epilogue_barrier(bool ok) {
  uint32_t all;
  __syncwarp();
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\nbar.red.and.pred q, 1, 128, p;\nselp.u32 %0, 1, 0, q;\n}"
               : "=r"(all) : "r"((uint32_t)ok) : "memory");
  return all != 0;
}

// A warp's 32 rows of a tile's accumulator, 32 columns at a time, to memory.  The loops are kept short and
// rolled up: written out straight, a tile's epilogue was three times as slow, waiting for its instructions.
struct Piece { uint32_t acc; int i0, j0, z, wide; bool mirror; };       // this warp's part of a tile
template <int KIND>
__device__ __forceinline__ void write_tile(const StepArgs &p, const CUtensorMap *rows_map, const CUtensorMap *cols_map, uint8_t *stage,
                                           const Piece &t, uint64_t *acc_empty) {
  const int lane = threadIdx.x & 31, i = t.i0 + lane, nc = KIND == kGram || KIND == kPoly ? p.m : p.n;
  const __half *D = p.A + t.z * p.ab + (long long)i * p.lda;
  uint4 ahead[4];            // kPoly: this lane's row of A, one piece of 32 columns ahead
  auto fetch = [&](int j) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
      ahead[c] = i < p.m && j + c * 8 < p.m ? *reinterpret_cast<const uint4 *>(D + j + c * 8) : make_uint4(0, 0, 0, 0);
  };
  if (KIND == kPoly) fetch(t.j0);
#pragma unroll 1
  for (int c0 = 0; c0 < t.wide; c0 += 32) {
    uint32_t v[32], q[16];
    tc_load32(t.acc + c0, v);
    uint8_t *rows = stage + ((c0 >> 5) & 1) * 4096, *cols = rows + 2048;
    if (KIND != kLast) {
      if (lane == 0) tc_store_read1();           // the buffer's last pieces have been read
      __syncwarp();
    }
    tc_wait_ld();
    if (c0 + 32 == t.wide) {                     // all of it is in registers: the tile after next may use the accumulator
      tc_fence_before();
      tc_warp_arrive(acc_empty);
    }
    const uint32_t *dd = reinterpret_cast<const uint32_t *>(ahead);
#pragma unroll
    for (int e = 0; e < 16; ++e)
      q[e] = finish<KIND>(p, __uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]), KIND == kPoly ? dd[e] : 0u, i, t.j0 + c0 + 2 * e);
    if (KIND == kPoly && c0 + 32 < t.wide) fetch(t.j0 + c0 + 32);
    const int j = t.j0 + c0;
    if (KIND != kLast) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<uint4 *>(rows + lane * 64 + ((c ^ (lane >> 1) & 3) << 4)) = make_uint4(q[4 * c], q[4 * c + 1], q[4 * c + 2], q[4 * c + 3]);
      if (t.mirror) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          uint16_t *to = reinterpret_cast<uint16_t *>(cols + 2 * e * 64 + (((lane >> 3) ^ (e & 3)) << 4)) + (lane & 7);
          to[0] = (uint16_t)(q[e] & 0xffffu);
          to[32] = (uint16_t)(q[e] >> 16);       // the next row, in the same place: the swizzle goes by pairs of rows
        }
      }
      tc_proxy_fence();
      __syncwarp();
      if (lane == 0) {
        if (t.i0 < p.m && j < nc) tc_store_3d(rows_map, smem_u32(rows), j, t.i0, t.z);
        if (t.mirror && t.i0 < p.m && j < nc) tc_store_3d(cols_map, smem_u32(cols), t.i0, j, t.z);
        tc_store_commit();
      }
    } else {
      const Out o = {static_cast<__half *>(p.o) + t.z * p.ob, p.os, p.tall ? p.n : p.m, p.tall ? p.m : p.n, p.vec != 0};
      if (p.tall) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          reinterpret_cast<uint16_t *>(rows)[(2 * e) * 40 + lane] = (uint16_t)(q[e] & 0xffffu);
          reinterpret_cast<uint16_t *>(rows)[(2 * e + 1) * 40 + lane] = (uint16_t)(q[e] >> 16);
        }
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) *reinterpret_cast<uint4 *>(rows + lane * 80 + c * 16) = make_uint4(q[4 * c], q[4 * c + 1], q[4 * c + 2], q[4 * c + 3]);
      }
      __syncwarp();
      put<32, 4>(reinterpret_cast<const __half *>(rows), 40, o, p.tall ? j : t.i0, p.tall ? t.i0 : j);
      __syncwarp();
    }
  }
}
// ... and, where the ranks of a cluster have parts of the sums, this warp's rows r0 .. r0 + SHARE - 1 of a tile:
// added up, finished and written
template <int KIND, int RANKS>
__device__ __forceinline__ void write_share(const StepArgs &p, uint32_t sums, __half *stage, int r0, int i0, int j0, int z, bool mirror) {
  constexpr int share = kM / RANKS / 4, pitch = 136;
  const int lane = threadIdx.x & 31;
  const __half *D = p.A + z * p.ab;
  __half *C = (KIND == kGram ? p.A : p.B) + z * p.ab;
#pragma unroll 4
  for (int k = 0; k < share; ++k) {              // a row of 128 values to a turn
    const int i = i0 + r0 + k, j = j0 + lane * 4;
    float4 y[RANKS];
#pragma unroll
    for (int o = 0; o < RANKS; ++o) y[o] = tc_peer_load(sums + sum_at(r0 + k, lane), o);
    uint2 d = make_uint2(0, 0);
    const bool inside = i < p.m && j < p.m;      // (rows of the workspace are padded to multiples of 8 values)
    if (KIND == kPoly && inside) d = *reinterpret_cast<const uint2 *>(D + (long long)i * p.lda + j);
    float4 x = y[0];
#pragma unroll
    for (int o = 1; o < RANKS; ++o) { x.x += y[o].x; x.y += y[o].y; x.z += y[o].z; x.w += y[o].w; }
    const uint2 h = make_uint2(finish<KIND>(p, x.x, x.y, d.x, i, j), finish<KIND>(p, x.z, x.w, d.y, i, j + 2));
    *reinterpret_cast<uint2 *>(stage + k * pitch + lane * 4) = h;
    if (inside) *reinterpret_cast<uint2 *>(C + (long long)i * p.lda + j) = h;
  }
  __syncwarp();
  if (!mirror) return;
#pragma unroll 2
  for (int k = lane; k < kM * (share / 8); k += 32) {           // transposed: pieces of eight rows
    const int c = k / (share / 8), rr = k % (share / 8) * 8;
    if (j0 + c >= p.m || i0 + r0 + rr >= p.m) continue;
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      o[e] = (uint32_t)__half_as_ushort(stage[(rr + 2 * e) * pitch + c]) | (uint32_t)__half_as_ushort(stage[(rr + 2 * e + 1) * pitch + c]) << 16;
    *reinterpret_cast<uint4 *>(C + (long long)(j0 + c) * p.lda + i0 + r0 + rr) = make_uint4(o[0], o[1], o[2], o[3]);
  }
  __syncwarp();
}

template <int BN, int RANKS>
__global__ void __launch_bounds__(kThreads, 1) orth_steps(const __grid_constant__ StepMaps maps, const StepArgs p) {
  typedef Shape<BN, RANKS> S;
  extern __shared__ __align__(1024) uint8_t base[];
  static_assert(sizeof(Bars<BN, RANKS>) <= 256 && S::smem <= 232448, "shared memory");
  Bars<BN, RANKS> &bar = *reinterpret_cast<Bars<BN, RANKS> *>(base + S::bars);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t ring = smem_u32(base);
  constexpr bool kSplit = RANKS > 1;
  const int rank = kSplit ? (int)tc_cluster_rank() : 0;
  const int cta = blockIdx.x, ctas = gridDim.x, cluster = cta / RANKS, clusters = ctas / RANKS;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::ring; ++s) { mbar_init(smem_u32(&bar.full[s]), 1); mbar_init(smem_u32(&bar.empty[s]), 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&bar.acc_full[s]), 1); mbar_init(smem_u32(&bar.acc_empty[s]), 4); }
    mbar_init(smem_u32(&bar.joined), 4 * RANKS);
    mbar_init(smem_u32(&bar.read), 4 * RANKS);
    mbar_init(smem_u32(&bar.finished), 1);
    mbar_init_fence();
  }
  if (warp == 1) tc_alloc(&bar.tmem, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t acc = bar.tmem;
  if (kSplit) tc_cluster_sync();            // the peers' barriers are ready
  cdg_grid_dep_wait();

  const int mt = (p.m + kM - 1) / kM, nt = (p.n + BN - 1) / BN, sym = mt * (mt + 1) / 2;
  // The products in turn.  A batch goes in two parts, of which one's products run while the other's are being
  // waited for.  The tiles are dealt out over the CTAs (or over the clusters, where those share the K loop) from
  // where the turn before ended, so that CTAs with a tile less in one turn have theirs first in the next.
  struct Turn { int kind, at, z0, tiles, nk, k0, dk, first, step; };       // at: which X is read
  const int parts = p.batch > 1 ? 2 : 1, turns = 3 * p.steps * parts;
  int dealt_to = 0;                        // the CTA that the next turn begins with
  auto turn_of = [&](int t) {
    Turn u;
    const int product = t / parts, which = product % 3, half = p.batch / 2;
    const int z0 = t % parts == 0 ? 0 : half, zn = parts == 1 ? p.batch : t % parts == 0 ? half : p.batch - half;
    u.at = (product / 3) & 1;
    u.kind = which < 2 ? which : product / 3 + 1 == p.steps ? kLast : kApply;
    u.z0 = z0;
    u.tiles = (which < 2 ? sym : mt * nt) * zn;
    const bool shared = kSplit && which < 2;
    const int steps = ((which == 0 ? p.n : p.m) + kK - 1) / kK;
    u.k0 = shared ? rank : 0;
    u.dk = shared ? RANKS : 1;
    u.nk = (steps - u.k0 + u.dk - 1) / u.dk;
    if (kSplit) {
      u.first = shared ? cluster : cta;
      u.step = shared ? clusters : ctas;
    } else {
      const int from = cta - dealt_to;
      u.first = from < 0 ? from + ctas : from;
      u.step = ctas;
      dealt_to = (dealt_to + u.tiles) % ctas;
    }
    return u;
  };
  struct Tile { int i0, j0, z; };
  auto tile_of = [&](const Turn &u, int at) {
    if (u.kind < 2) {        // tiles (i, j), i <= j, counted column by column
      const int z = at / sym, t = at % sym;
      int j = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
      while ((j + 1) * (j + 2) / 2 <= t) ++j;
      while (j * (j + 1) / 2 > t) --j;
      return Tile{(t - j * (j + 1) / 2) * kM, j * kM, u.z0 + z};
    }
    const int z = at / (mt * nt), t = at % (mt * nt);
    return Tile{t % mt * kM, t / mt * BN, u.z0 + z};
  };

  if (warp == 0) {
    if (tc_elect()) {
      bool ok = true;
      int n = 0;
      for (int t = 0; t < turns && ok; ++t) {
        const Turn u = turn_of(t);
        long long deadline = clock64() + p.wait;
        if (t >= parts && u.first < u.tiles) {         // every CTA has written its share of this part's product before
          if (!(ok = wait_count(p.arrived + t % parts, (unsigned)(t / parts) * (unsigned)ctas, deadline))) break;
          asm volatile("fence.proxy.async;" ::: "memory");         // ... and the copies see it
        }
        const CUtensorMap *ma = u.kind == kGram ? &maps.rows[u.at] : u.kind == kPoly ? &maps.A : &maps.B;
        const CUtensorMap *mb = u.kind == kGram ? &maps.rows[u.at] : u.kind == kPoly ? &maps.A : &maps.panels[u.at];
        for (int at = u.first; at < u.tiles && ok; at += u.step) {
          const Tile w = tile_of(u, at);
          deadline = clock64() + p.wait;
          for (int it = 0; it < u.nk; ++it, ++n) {
            if (!(ok = tc_wait_released(bar.empty, n, S::ring, deadline))) break;
            const uint32_t full = smem_u32(&bar.full[n % S::ring]), a = ring + n % S::ring * S::stage, b = a + S::a_bytes;
            const int k0 = (u.k0 + it * u.dk) * kK;
            mbar_expect_tx(full, u.kind < 2 ? 2 * S::a_bytes : S::stage);
            tma_load_3d(a, ma, k0, w.i0, w.z, full);
            if (u.kind < 2) {
              tma_load_3d(b, mb, k0, w.j0, w.z, full);
            } else {           // panels of 64 columns, 64 rows of K
#pragma unroll
              for (int c = 0; c < BN / 64; ++c) tma_load_3d(b + c * kK * 128, mb, w.j0 + c * 64, k0, w.z, full);
            }
          }
        }
      }
      if (!ok) atomicOr(p.status, CDG_ST_TIMEOUT);
      tc_drain(bar.full, n, S::ring);
    }
  } else if (warp == 1) {
    bool ok = true;
    int n = 0, seq = 0;
    for (int t = 0; t < turns && ok; ++t) {
      const Turn u = turn_of(t);
      const uint32_t idesc = u.kind < 2 ? tc_idesc(false, kM, kM, false, false) : tc_idesc(false, kM, BN, false, true);
      const uint32_t kb = u.kind < 2 ? 2 : 128;          // 16 of K further on in B, in units of 16 bytes
      for (int at = u.first; at < u.tiles && ok; at += u.step, ++seq) {
        const long long deadline = clock64() + 2 * p.wait;       // (the copies may wait for the grid)
        const uint32_t d = acc + (seq & 1) * 256;
        if (seq >= 2 && !(ok = tc_wait(&bar.acc_empty[seq & 1], tc_parity(seq - 2, 2), deadline))) break;
        for (int it = 0; it < u.nk; ++it, ++n) {
          if (!(ok = tc_wait(&bar.full[n % S::ring], tc_parity(n, S::ring), deadline))) break;
          tc_fence_after();
          const uint32_t a = ring + n % S::ring * S::stage, b = a + S::a_bytes;
          const uint64_t da = tc_desc_k(a), db = u.kind < 2 ? tc_desc_k(b) : tc_desc_mn(b, kK * 128);
          if (tc_elect()) {
#pragma unroll
            for (int kk = 0; kk < kK / 16; ++kk) tc_mma(d, da + kk * 2, db + kk * kb, idesc, it > 0 || kk > 0);
            tc_commit(&bar.empty[n % S::ring]);
          }
          __syncwarp();
        }
        if (!ok) break;
        if (tc_elect()) tc_commit(&bar.acc_full[seq & 1]);
        __syncwarp();
      }
    }
    if (!ok && lane == 0) atomicOr(p.status, CDG_ST_TIMEOUT);
    tc_finish(&bar.finished);
  } else {
    const int w = warp & 3, r = w * 32 + lane;         // warp w of the four reads lanes 32 w ... of the accumulator
    uint8_t *stage = base + S::staging + w * S::warp_bytes;
    bool ok = true;
    int seq = 0, joins = 0;
    for (int t = 0; t < turns && ok; ++t) {
      const Turn u = turn_of(t);
      const bool split = kSplit && u.kind < 2;
      if (u.kind == kPoly && u.first < u.tiles) {      // A, which is added, is read here too
        ok = lane != 0 || wait_count(p.arrived + t % parts, (unsigned)(t / parts) * (unsigned)ctas, clock64() + 2 * p.wait);
        __syncwarp();            // lane 0 has acquired the other CTAs' writes: the lanes' reads come after that (a vote orders no memory)
        ok = __all_sync(0xffffffffu, ok);
      }
      for (int at = u.first; at < u.tiles && ok; at += u.step, ++seq) {
        const Tile tile = tile_of(u, at);
        const long long deadline = clock64() + 3 * p.wait;
        const Piece piece = {acc + ((uint32_t)(w * 32) << 16) + (seq & 1) * 256, tile.i0 + w * 32, tile.j0, tile.z, u.kind < 2 ? kM : BN,
                             u.kind < 2 && tile.i0 != tile.j0};
        uint64_t *empty = &bar.acc_empty[seq & 1];
        if (!(ok = tc_wait(&bar.acc_full[seq & 1], tc_parity(seq, 2), deadline))) break;
        tc_fence_after();
        if (!split) {
          if (u.kind == kGram) write_tile<kGram>(p, &maps.to_A, &maps.to_A, stage, piece, empty);
          else if (u.kind == kPoly) write_tile<kPoly>(p, &maps.to_B, &maps.to_B, stage, piece, empty);
          else if (u.kind == kApply) write_tile<kApply>(p, &maps.to_x[1 - u.at], nullptr, stage, piece, empty);
          else write_tile<kLast>(p, nullptr, nullptr, stage, piece, empty);
          continue;
        }
        // this CTA's sums, after the peers have read those of the tile before
        if (joins > 0 && !(ok = tc_wait_cluster(&bar.read, (joins - 1) & 1, deadline))) break;
#pragma unroll 1
        for (int c0 = 0; c0 < kM; c0 += 32) {
          uint32_t v[32];
          tc_load32(piece.acc + c0, v);
          tc_wait_ld();
#pragma unroll
          for (int i = 0; i < 8; ++i)            // (every rank has had two steps of K at least)
            *reinterpret_cast<uint4 *>(base + S::sums + sum_at(r, (c0 >> 2) + i)) = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        }
        tc_fence_before();
        tc_warp_arrive(empty);
        if (lane < RANKS) tc_arrive_peer(&bar.joined, lane);
        if (!(ok = tc_wait_cluster(&bar.joined, joins & 1, deadline))) break;
        ++joins;
        const int r0 = rank * (kM / RANKS) + w * (kM / RANKS / 4);
        __half *mine = reinterpret_cast<__half *>(stage);
        if (u.kind == kGram) write_share<kGram, RANKS>(p, ring + S::sums, mine, r0, tile.i0, tile.j0, tile.z, piece.mirror);
        else write_share<kPoly, RANKS>(p, ring + S::sums, mine, r0, tile.i0, tile.j0, tile.z, piece.mirror);
        if (lane < RANKS) tc_arrive_peer(&bar.read, lane);
      }
      if (t + parts < turns) {
        // this CTA's share is written (by lane 0's copies, or by all lanes): visible to all, then counted; one
        // without a share is counted no earlier than the product before is complete, so that the count tells
        unsigned *count = p.arrived + t % parts;
        if (lane == 0) tc_store_done();
        if (split || lane == 0) asm volatile("fence.proxy.async;" ::: "memory");
        if (threadIdx.x == 64 && u.first >= u.tiles && t >= parts)
          ok = wait_count(count, (unsigned)(t / parts) * (unsigned)ctas, clock64() + 2 * p.wait);
        ok = epilogue_barrier(ok);       // (a warp that left alone would keep the others at this barrier for good)
        if (ok && threadIdx.x == 64) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(count) : "memory");
      }
    }
    if (lane == 0) tc_store_done();
    if (!ok && lane == 0) atomicOr(p.status, CDG_ST_TIMEOUT);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) { tc_fence_after(); tc_free(acc, 512); }
  if (kSplit) tc_cluster_sync();            // no CTA leaves while another reads its sums
}

// ---- small matrices -----------------------------------------------------------------------------
// Up to 128 x 576: X, A and B stay in one CTA's shared memory for all steps, one CTA to a matrix and one launch in
// all.  X lies in panels of 64 columns (128 rows of 128 bytes, swizzled), which serve as they are as the K-major
// operands of X X^T and as the MN-major one of B X; a block of 128 columns of X is replaced where it lies when
// its product is over.
constexpr int kSmallThreads = 512, kSmallCols = 576;         // (eight of the warps read accumulators, all move G and O)
constexpr uint32_t kPanel = 16384;
inline size_t small_smem(int n) { return (size_t)((n + 63) / 64 + 4) * kPanel + 1024; }       // 1024: to a boundary of the swizzle

struct SmallArgs {
  int rows, cols, tall, steps, vec;
  float a, b, c, eps;
  long long gb, gs, ob, os, wait;                // wait: how long one may last, in clock cycles
  int *status;
};

// where 8 values from column c (a multiple of 8) of row r lie
__device__ __forceinline__ uint32_t small_at(int r, int c) { return (uint32_t)(c >> 6) * kPanel + r * 128 + ((((c >> 3) ^ r) & 7) << 4); }

template <typename T, int VEC>
__global__ void __launch_bounds__(kSmallThreads, 1) orth_small(const T *g, __nv_bfloat16 *o, const SmallArgs p) {
  extern __shared__ __align__(16) uint8_t dyn[];
  uint8_t *const base = dyn + ((1024u - (smem_u32(dyn) & 1023u)) & 1023u);
  __shared__ double part[kSmallThreads / 32];
  __shared__ __align__(8) uint64_t bar[5];         // A and A A; three blocks of X; the end
  __shared__ uint32_t slot;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int m = p.tall ? p.cols : p.rows, n = p.tall ? p.rows : p.cols, panels = (n + 63) / 64;
  uint8_t *A = base + panels * kPanel, *B = A + 2 * kPanel;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 5; ++i) mbar_init(smem_u32(&bar[i]), 1);
    mbar_init_fence();
  }
  if (warp == 0) tc_alloc(&slot, 512);
  for (uint32_t i = threadIdx.x * 16; i < panels * kPanel; i += kSmallThreads * 16) *reinterpret_cast<uint4 *>(base + i) = make_uint4(0, 0, 0, 0);
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  g += blockIdx.x * p.gb;
  o += blockIdx.x * p.ob;

  // X = kScale G / (|G| + eps); G twice, the second time out of L2, VEC values to a load and eight loads at a time
  struct __align__(sizeof(T) * VEC) Load { T v[VEC]; };
  const int per = p.cols / VEC, all = p.rows * per;
  auto each = [&](auto &&use) {
    for (int i = threadIdx.x; i < all; i += 8 * kSmallThreads) {
      Load q[8];
      int r[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int at = i + k * kSmallThreads;
        r[k] = at / per;
        if (at < all) q[k] = *reinterpret_cast<const Load *>(g + (long long)r[k] * p.gs + (at - r[k] * per) * VEC);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int at = i + k * kSmallThreads;
        if (at < all) use(r[k], (at - r[k] * per) * VEC, q[k]);
      }
    }
  };
  double s = 0.0;
  each([&](int, int, const Load &q) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) { const double v = cdg_ld(&q.v[e]); s = fma(v, v, s); }
  });
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
  if (lane == 0) part[warp] = s;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  s = 0.0;
  for (int i = 0; i < kSmallThreads / 32; ++i) s += part[i];
  const double norm = sqrt(s) + (double)p.eps;
  const float f = norm > 0.0 ? (float)fmin((double)kScale / norm, 3e38) : 0.0f;
  each([&](int gr, int gc, const Load &q) {
    struct __align__(2 * VEC) Halves { __half v[VEC]; } h;
#pragma unroll
    for (int e = 0; e < VEC; ++e) h.v[e] = __float2half_rn(f * cdg_ld(&q.v[e]));
    if (p.tall) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) *reinterpret_cast<__half *>(base + small_at(gc + e, gr & ~7) + (gr & 7) * 2) = h.v[e];
    } else {
      *reinterpret_cast<Halves *>(base + small_at(gr, gc & ~7) + (gc & 7) * 2) = h;
    }
  });
  tc_proxy_fence();
  __syncthreads();

  const uint32_t tm = slot, mine = tm + ((uint32_t)((warp & 3) * 32) << 16);
  const uint32_t sx = smem_u32(base), sa = smem_u32(A), sb = smem_u32(B);
  const int r = (warp & 3) * 32 + lane, half = warp >> 2;          // (warps 8 to 15: half 2 and 3, none of the columns)
  bool ok = true;
  uint32_t turn[4] = {0, 0, 0, 0};             // phases of the barriers
  // products whose K index runs along the rows of both operands, `panels_` panels of 64
  auto gram = [&](uint32_t x, int panels_) {
    if (warp == 0) {
      if (tc_elect()) {
        constexpr uint32_t idesc = tc_idesc(false, 128, 128, false, false);
        const uint64_t d = tc_desc_k(x);
        for (int q = 0; q < panels_; ++q)
#pragma unroll
          for (int k = 0; k < 4; ++k) tc_mma(tm, d + q * (kPanel >> 4) + k * 2, d + q * (kPanel >> 4) + k * 2, idesc, q > 0 || k > 0);
        tc_commit(&bar[0]);
      }
      __syncwarp();
    }
    ok = tc_wait(&bar[0], turn[0]++ & 1, clock64() + p.wait);
    tc_fence_after();
  };
  auto settle = [&]() {          // what was written is an operand of the next product, what was read may be overwritten
    tc_proxy_fence();
    tc_fence_before();
    ok = __syncthreads_and(ok);
    tc_fence_after();
  };
  for (int step = 0; step < p.steps && ok; ++step) {
    const bool last = step + 1 == p.steps;
    gram(sx, panels);
#pragma unroll 1
    for (int c0 = half * 64; c0 < half * 64 + 64 && half < 2; c0 += 32) {
      uint32_t v[32];
      tc_load32(mine + c0, v);
      tc_wait_ld();
#pragma unroll
      for (int c = 0; c < 32; c += 8) {
        uint32_t q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const __half2 h = __floats2half2_rn(__uint_as_float(v[c + 2 * e]) * (1.0f / (kScale * kScale)), __uint_as_float(v[c + 2 * e + 1]) * (1.0f / (kScale * kScale)));
          q[e] = *reinterpret_cast<const uint32_t *>(&h);
        }
        *reinterpret_cast<uint4 *>(A + small_at(r, c0 + c)) = make_uint4(q[0], q[1], q[2], q[3]);
      }
    }
    settle();
    if (!ok) break;
    gram(sa, 2);
#pragma unroll 1
    for (int c0 = half * 64; c0 < half * 64 + 64 && half < 2; c0 += 32) {
      uint32_t v[32];
      tc_load32(mine + c0, v);
      tc_wait_ld();
#pragma unroll
      for (int c = 0; c < 32; c += 8) {
        const uint4 x = *reinterpret_cast<const uint4 *>(A + small_at(r, c0 + c));
        const uint32_t d[4] = {x.x, x.y, x.z, x.w};
        uint32_t q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 w = __half22float2(*reinterpret_cast<const __half2 *>(&d[e]));
          const int j = c0 + c + 2 * e;
          const __half2 h = __floats2half2_rn(fmaf(p.b, w.x, __uint_as_float(v[c + 2 * e]) * p.c) + (r == j ? p.a : 0.0f),
                                              fmaf(p.b, w.y, __uint_as_float(v[c + 2 * e + 1]) * p.c) + (r == j + 1 ? p.a : 0.0f));
          q[e] = *reinterpret_cast<const uint32_t *>(&h);
        }
        *reinterpret_cast<uint4 *>(B + small_at(r, c0 + c)) = make_uint4(q[0], q[1], q[2], q[3]);
      }
    }
    settle();
    if (!ok) break;
    for (int q0 = 0; q0 < panels && ok; q0 += 6) {           // three blocks of 128 columns at a time
      if (warp == 0) {
        if (tc_elect()) {
          for (int q = q0; q < panels && q < q0 + 6; q += 2) {
            const uint32_t idesc = tc_idesc(false, 128, q + 1 < panels ? 128 : 64, false, true);
            const uint64_t da = tc_desc_k(sb), db = tc_desc_mn(sx + q * kPanel, kPanel);
#pragma unroll
            for (int k = 0; k < 8; ++k) tc_mma(tm + 128 + (q - q0) * 64, da + (k >> 2) * (kPanel >> 4) + (k & 3) * 2, db + k * 128, idesc, k > 0);
            tc_commit(&bar[1 + (q - q0) / 2]);
          }
        }
        __syncwarp();
      }
#pragma unroll
      for (int t = 0; t < 3; ++t) {
        const int q = q0 + 2 * t;
        if (q >= panels || !ok) continue;
        if (!(ok = tc_wait(&bar[1 + t], turn[1 + t]++ & 1, clock64() + p.wait))) continue;
        tc_fence_after();
        if (half > 1 || q + half >= panels) continue;
#pragma unroll 1
        for (int c0 = half * 64; c0 < half * 64 + 64; c0 += 32) {
          uint32_t v[32];
          tc_load32(mine + 128 + t * 128 + c0, v);
          tc_wait_ld();
          const int j = q * 64 + c0;
#pragma unroll
          for (int c = 0; c < 32; c += 8) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x = __uint_as_float(v[c + 2 * e]), y = __uint_as_float(v[c + 2 * e + 1]);
              if (last) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(x * (1.0f / kScale), y * (1.0f / kScale));
                w[e] = *reinterpret_cast<const uint32_t *>(&h);
              } else {
                const __half2 h = __floats2half2_rn(x, y);
                w[e] = *reinterpret_cast<const uint32_t *>(&h);
              }
            }
            *reinterpret_cast<uint4 *>(base + small_at(r, j + c)) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
      settle();
    }
  }
  // O, rows of it in pieces of eight values, out of X's place
  const int pieces = (p.cols + 7) / 8;
  for (int i = threadIdx.x; i < p.rows * pieces && ok; i += kSmallThreads) {
    const int orow = i / pieces, c0 = (i - orow * pieces) * 8;
    __nv_bfloat16 *to = o + (long long)orow * p.os + c0;
    uint32_t w[4];
    if (p.tall) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint8_t *at = base + (orow & 7) * 2;
        const int r0 = c0 + 2 * e;                // (rows up to 127 are there)
        w[e] = (uint32_t)*reinterpret_cast<const uint16_t *>(at + small_at(r0, orow & ~7)) |
               (uint32_t)*reinterpret_cast<const uint16_t *>(at + small_at(r0 + 1, orow & ~7)) << 16;
      }
    } else {
      const uint4 x = *reinterpret_cast<const uint4 *>(base + small_at(orow, c0));
      w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
    }
    if (p.vec && c0 + 8 <= p.cols) {
      *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c0 + e < p.cols) to[e] = __ushort_as_bfloat16((unsigned short)(w[e >> 1] >> (16 * (e & 1))));
    }
  }
  if (!ok && threadIdx.x == 0) atomicOr(p.status, CDG_ST_TIMEOUT);
  if (warp == 0) tc_finish(&bar[4]);
  tc_fence_before();
  __syncthreads();
  if (warp == 0) { tc_fence_after(); tc_free(tm, 512); }
}

// Whether X (times kScale), A and B stay within fp16 (65504) for these coefficients.  An entry is no larger than the
// largest singular value.  Those of X start in [0, 1] and go through s (a + b s^2 + c s^4), so they stay below the
// largest magnitude of that on [0, top], step by step: at an end or where the derivative a + 3 b t + 5 c t^2 is zero
// (t = s^2).  Roundings are allowed 2^-8 a step.  A has their squares, and B the magnitudes of a + b t + c t^2, largest
// at an end or at t = -b / 2c.
bool in_range(const float *coeffs, int steps) {
  const double a = coeffs[0], b = coeffs[1], c = coeffs[2], slack = 1.0 + 1.0 / 256, most = 60000.0;
  double top = slack;
  for (int i = 0; i < steps; ++i) {
    if (!(top * kScale <= most)) return false;            // (then A's entries, up to top squared, are in range too)
    const double end = top * top;
    double x = 0.0, y = fabs(a);
    const auto at = [&](double t) {
      if (!(t > 0.0 && t <= end)) return;
      const double f = fabs(a + t * (b + t * c));
      x = fmax(x, sqrt(t) * f);
      y = fmax(y, f);
    };
    at(end);
    if (c != 0.0) {
      const double root = 9.0 * b * b - 20.0 * a * c;
      at(-b / (2.0 * c));
      if (root >= 0.0) { at((-3.0 * b + sqrt(root)) / (10.0 * c)); at((-3.0 * b - sqrt(root)) / (10.0 * c)); }
    } else if (b != 0.0) {
      at(-a / (3.0 * b));
    }
    if (!(y <= most)) return false;
    top = x * slack;                                      // (the last X is written as bf16)
  }
  return true;
}

constexpr long long kMaxStride = 1ll << 38;   // elements, as for attention: products with a row number stay below 2^63
inline long long up(long long v, long long to) { return (v + to - 1) / to * to; }

struct Plan {
  int m, n, ldx, lda;
  long long part, arrived, x0, x1, a, b, total;    // byte offsets in the workspace
};
Plan plan_of(long long batch, int rows, int cols) {
  Plan p;
  p.m = rows < cols ? rows : cols;
  p.n = rows < cols ? cols : rows;
  p.ldx = (int)up(p.n, 8);
  p.lda = (int)up(p.m, 8);
  const long long xb = up(2 * batch * p.m * p.ldx, 256), ab = up(2 * batch * p.m * p.lda, 256);
  p.part = 0;
  p.arrived = 8 * batch * kNormBlocks;
  p.x0 = up(p.arrived + 8, 256);
  p.x1 = p.x0 + xb;
  p.a = p.x1 + xb;
  p.b = p.a + ab;
  p.total = p.b + ab;
  return p;
}

template <int BN, int RANKS>
int launch(const StepMaps &maps, const StepArgs &a, int sms, int device, cudaStream_t st) {
  static CdgPerDevice flags;
  static std::atomic<int> room[64];           // CTAs that are resident at once, by device
  if (!tc_raise_limit(flags, orth_steps<BN, RANKS>, Shape<BN, RANKS>::smem)) return CDGRAB_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = RANKS;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeCooperative;             // all CTAs at once: they wait for one another
  at[1].val.cooperative = 1;
  cfg.gridDim = dim3(sms / RANKS * RANKS); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = Shape<BN, RANKS>::smem; cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  int n = device < 64 ? room[device].load(std::memory_order_relaxed) : 0;
  if (n == 0) {
    if (RANKS == 1) n = sms;
    else if (cudaOccupancyMaxActiveClusters(&n, orth_steps<BN, RANKS>, &cfg) != cudaSuccess || n < 1) return cdg_launch_rc(cudaErrorUnknown);
    else n = n * RANKS < sms ? n * RANKS : sms / RANKS * RANKS;
    if (device < 64) room[device].store(n, std::memory_order_relaxed);
  }
  cfg.gridDim = dim3(n);
  cfg.numAttrs = 2;
  return cdg_launch_rc(cudaLaunchKernelEx(&cfg, orth_steps<BN, RANKS>, maps, a));
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
  if (need < 0 || (long long)rows * cols / (64 * 64) * (batch > 0 ? batch : 1) > (1 << 28) || steps < 1 || steps > 64 || !coeffs || !(eps >= 0.0f) || (dtype != CDGRAB_F32 && dtype != CDGRAB_BF16))
    return CDGRAB_ERR_INVALID;
  if (!isfinite(coeffs[0]) || !isfinite(coeffs[1]) || !isfinite(coeffs[2])) return CDGRAB_ERR_INVALID;
  if (batch == 0 || rows == 0 || cols == 0) return CDGRAB_OK;
  if (!in_range(coeffs, steps)) return CDGRAB_ERR_INVALID;
  if (!g || !o || !workspace || workspace_bytes < need || !cdg_aligned(workspace, 16) || gs < cols || os < cols ||
      gs > kMaxStride || os > kMaxStride || (batch > 1 && (gb < 0 || ob < (long long)(rows - 1) * os + cols)))
    return CDGRAB_ERR_INVALID;
  if (!cdg_aligned(g, dtype == CDGRAB_F32 ? 4 : 2) || !cdg_aligned(o, 2)) return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const Plan p = plan_of(batch, rows, cols);
  const int tall = rows > cols, m = p.m, n = p.n;
  const int e = dtype == CDGRAB_F32 ? 4 : 2;
  const bool wide = cdg_aligned(g, 16) && gs % (16 / e) == 0 && gb % (16 / e) == 0 && cols % (16 / e) == 0;
  if (m <= 128 && n <= kSmallCols) {
    const SmallArgs a = {rows, cols, tall, steps, cdg_aligned(o, 16) && os % 8 == 0 && ob % 8 == 0, coeffs[0], coeffs[1], coeffs[2], eps, gb, gs, ob, os,
                         cdg_ops_wait_limit(), dev->status};
    auto run = [&](auto *kernel, const auto *from, CdgPerDevice &flags) {
      if (!tc_raise_limit(flags, kernel, small_smem(kSmallCols))) return (int)CDGRAB_ERR_CUDA;
      return cdg_launch_rc(cdg_ops_launch(kernel, dim3(batch), kSmallThreads, small_smem(n), st, from, (__nv_bfloat16 *)o, a));
    };
    static CdgPerDevice flags[4];
    if (dtype == CDGRAB_F32)
      return wide ? run(orth_small<float, 4>, (const float *)g, flags[0]) : run(orth_small<float, 1>, (const float *)g, flags[1]);
    return wide ? run(orth_small<__nv_bfloat16, 8>, (const __nv_bfloat16 *)g, flags[2])
                : run(orth_small<__nv_bfloat16, 1>, (const __nv_bfloat16 *)g, flags[3]);
  }
  char *w = (char *)up((long long)(uintptr_t)workspace, 256);
  double *part = (double *)(w + p.part);
  unsigned *arrived = (unsigned *)(w + p.arrived);
  __half *x[2] = {(__half *)(w + p.x0), (__half *)(w + p.x1)}, *A = (__half *)(w + p.a), *B = (__half *)(w + p.b);
  const long long xb = (long long)m * p.ldx, ab = (long long)m * p.lda;

  StepMaps maps;
  const long long dx[3] = {n, m, batch}, sx[3] = {1, p.ldx, xb}, da[3] = {m, m, batch}, sa[3] = {1, p.lda, ab};
  for (int i = 0; i < 2; ++i)
    if (!tc_encode(&maps.rows[i], false, x[i], 3, dx, sx, kM) || !tc_encode(&maps.panels[i], false, x[i], 3, dx, sx, kK)) return CDGRAB_ERR_CUDA;
  for (int i = 0; i < 2; ++i)
    if (!tc_encode(&maps.to_x[i], false, x[i], 3, dx, sx, 32, 32)) return CDGRAB_ERR_CUDA;
  if (!tc_encode(&maps.A, false, A, 3, da, sa, kM) || !tc_encode(&maps.B, false, B, 3, da, sa, kM) ||
      !tc_encode(&maps.to_A, false, A, 3, da, sa, 32, 32) || !tc_encode(&maps.to_B, false, B, 3, da, sa, 32, 32))
    return CDGRAB_ERR_CUDA;

  const dim3 gt((cols + 63) / 64, (rows + 63) / 64, batch);
  int rc;
  auto begin = [&](auto *sumsq, auto *start, const auto *from) {
    const int r = cdg_launch_rc(cdg_ops_launch(sumsq, dim3(kNormBlocks, batch), 256, 0, st, from, gb, gs, rows, cols, part, arrived));
    return r != CDGRAB_OK ? r : cdg_launch_rc(cdg_ops_launch(start, gt, 256, 0, st, from, gb, gs, rows, cols, tall, part, eps, x[0], p.ldx, xb));
  };
  if (dtype == CDGRAB_F32)
    rc = wide ? begin(orth_sumsq<float, 4>, orth_start<float, 4>, (const float *)g) : begin(orth_sumsq<float, 1>, orth_start<float, 1>, (const float *)g);
  else
    rc = wide ? begin(orth_sumsq<__nv_bfloat16, 8>, orth_start<__nv_bfloat16, 8>, (const __nv_bfloat16 *)g)
              : begin(orth_sumsq<__nv_bfloat16, 1>, orth_start<__nv_bfloat16, 1>, (const __nv_bfloat16 *)g);
  if (rc != CDGRAB_OK) return rc;
  const StepArgs a = {m, n, batch, steps, p.ldx, p.lda, tall, cdg_aligned(o, 16) && os % 8 == 0 && ob % 8 == 0, coeffs[0], coeffs[1], coeffs[2],
                      {x[0], x[1]}, A, B, o, xb, ab, ob, os, arrived, cdg_ops_wait_limit(), dev->status};
  // tiles of 256 columns while they still give every SM one; CTAs share a tile of A or B where there are fewer
  // than half as many tiles as SMs, up to four of them and at least two steps of K each
  const long long mt = (m + kM - 1) / kM, sym = mt * (mt + 1) / 2 * batch;
  if (mt * ((n + 255) / 256) * batch >= dev->sms) return launch<256, 1>(maps, a, dev->sms, dev->index, st);
  const int k = (m + kK - 1) / kK;
  if (sym * 4 <= dev->sms && k >= 8) return launch<128, 4>(maps, a, dev->sms, dev->index, st);
  if (sym * 2 <= dev->sms && k >= 4) return launch<128, 2>(maps, a, dev->sms, dev->index, st);
  return launch<128, 1>(maps, a, dev->sms, dev->index, st);
}
