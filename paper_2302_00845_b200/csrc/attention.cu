// Softmax attention, forward and backward, on the 5th-generation tensor cores: bf16 operands, 32-bit sums.
//
// Forward:   s = scale q k^T,  lse = log sum_j exp(s_j),  o = sum_j exp(s_j - lse) v_j.
// Backward:  p = exp(s - lse),  delta = sum_d do o,  ds = p (do v^T - delta),
//            dq = scale ds k,  dk = scale ds^T q,  dv = p^T do  (dk, dv summed over the query heads of a key head).
//
// Common to the three kernels: tiles of 128 x 128 scores.  A bulk-copy warp fills rings of shared-memory
// tiles (panels of 64 head dimensions, 128-byte swizzle, zeros past the tensor's ends), a matrix warp
// issues the products, and the other warps read scores from tensor memory, one row per thread, and write
// probabilities (or their gradients) back to it as the bf16 operand of the next product.  Nothing of the
// size of the score matrix ever leaves the SM.  Rounding a probability to bf16 changes it by at most
// 2^-8 relative, as much as the output's own rounding; running maxima, sums and accumulators are fp32.
//
// Masking: a score outside the visible set is replaced, not added to, so whatever lies there (NaN
// included) is never used; rows of a tile past a sequence's length are zeroed in shared memory where they
// are the summed index of a product, because 0 x NaN would not be 0.
#include <math.h>

#include "tensor_core.cuh"

namespace {

typedef __nv_bfloat16 bf16;

constexpr int kT = 128;                       // edge of a score tile
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Sizes {
  int batch, tq, tk, heads, group, dim, causal;
  float scale;               // as given
  float a;                   // |scale| log2 e, at least 1e-30: a scale of 0 still leaves masked scores at -infinity
  int negative;              // scale < 0
  int shared;                // bits q, k, v, do: one for the whole batch (a batch stride of 0)
  const int *q_lens, *kv_lens;
  long long wait;            // how long the waits of one block of rows may last, in clock cycles
  int *status;
};
struct View { bf16 *p; long long b, t, h; };

enum { kQ = 1, kK = 2, kV = 4, kDo = 8 };
__device__ __forceinline__ int batch_of(const Sizes &z, int which, int b) { return z.shared & which ? 0 : b; }
__device__ __forceinline__ int used(const int *lens, int b, int most) { return lens ? min(max(lens[b], 0), most) : most; }
// (the special function units do 16 a cycle and SM, 1024 cycles for a tile of 128 x 128; a quarter of them as
// polynomials on the FMA units made no kernel here faster)
__device__ __forceinline__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float2 exp2_two(float2 x) { return make_float2(exp2_fast(x.x), exp2_fast(x.y)); }
__device__ __forceinline__ float2 two(const uint32_t (&v)[2][32], int e) {
  return make_float2(__uint_as_float(v[e >> 5][e & 31]), __uint_as_float(v[e >> 5][(e & 31) + 1]));
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&h);
}

// one tile of 128 tokens of one head: NP panels of 64 head dimensions
template <int NP>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap *map, int token, int head, int batch, uint32_t bar) {
#pragma unroll
  for (int p = 0; p < NP; ++p) tma_load_4d(dst + p * kT * 128, map, p * 64, token, head, batch, bar);
}
// zeroes rows from..127 of a tile (a whole warp)
template <int NP>
__device__ __forceinline__ void zero_rows(uint8_t *tile, int from) {
  const int lane = threadIdx.x & 31;
  for (int r = from + (lane >> 3); r < kT; r += 4)
#pragma unroll
    for (int p = 0; p < NP; ++p) *reinterpret_cast<uint4 *>(tile + p * kT * 128 + r * 128 + (lane & 7) * 16) = make_uint4(0, 0, 0, 0);
  tc_proxy_fence();
  __syncwarp();
}

// products of one tile, issued by one thread.  128-row operands, DP = 64 NP head dimensions.
// scores: D[128][128] = A B^T over the head dimension
template <int NP>
__device__ __forceinline__ void mma_scores(uint32_t d, uint32_t a, uint32_t b) {
  constexpr uint32_t idesc = tc_idesc(true, kT, kT, false, false);
  const uint64_t da = tc_desc_k(a), db = tc_desc_k(b);          // addresses in units of 16 bytes
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int k = 0; k < 4; ++k) tc_mma(d, da + (p * kT * 8 + k * 2), db + (p * kT * 8 + k * 2), idesc, p > 0 || k > 0);
}
// weighted rows: D[128][DP] (+)= W B, W a 128 x 128 bf16 operand in tensor memory whose columns 64..127
// start `half` 32-bit columns after the first, B 128 rows of DP values
template <int NP>
__device__ __forceinline__ void mma_rows(uint32_t d, uint32_t w, uint32_t half, uint32_t b, bool add) {
  constexpr uint32_t idesc = tc_idesc(true, kT, 64 * NP, false, true);
  const uint64_t db = tc_desc_mn(b, kT * 128);
#pragma unroll
  for (int k = 0; k < 8; ++k) tc_mma_ta(d, w + (k >> 2) * half + (k & 3) * 8, db + k * 128, idesc, add || k > 0);
}

// 32 rows of DP bf16 values from registers to memory through this warp's part of a tile: each lane
// brings its row, the warp writes whole rows
template <int NP>
__device__ __forceinline__ void stage_row(uint8_t *tile, int row, int c0, const uint32_t (&w)[16]) {   // 32 values from column c0
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int chunk = (c0 >> 3) + i;
    *reinterpret_cast<uint4 *>(tile + (chunk >> 3) * kT * 128 + row * 128 + (((chunk & 7) ^ (row & 7)) << 4)) =
        make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
}
// `rows` staged rows from row0 on (a whole warp)
template <int NP>
__device__ __forceinline__ void write_rows(const uint8_t *tile, int row0, int rows, int token0, int tokens, const Sizes &z, bf16 *dst, long long stride) {
  const int lane = threadIdx.x & 31, per = NP * 8;
  for (int i = lane; i < rows * per; i += 32) {
    const int r = row0 + i / per, chunk = i % per;
    if (token0 + r < tokens && chunk * 8 < z.dim)
      *reinterpret_cast<uint4 *>(dst + (long long)(token0 + r) * stride + chunk * 8) =
          *reinterpret_cast<const uint4 *>(tile + (chunk >> 3) * kT * 128 + r * 128 + (((chunk & 7) ^ (r & 7)) << 4));
  }
}
// ... and rows of zeros
template <int NP>
__device__ __forceinline__ void write_zeros(int row0, int rows, int token0, int tokens, const Sizes &z, bf16 *dst, long long stride) {
  const int lane = threadIdx.x & 31, per = NP * 8;
  for (int i = lane; i < rows * per; i += 32) {
    const int r = row0 + i / per, chunk = i % per;
    if (token0 + r < tokens && chunk * 8 < z.dim)
      *reinterpret_cast<uint4 *>(dst + (long long)(token0 + r) * stride + chunk * 8) = make_uint4(0, 0, 0, 0);
  }
}

// All three kernels are persistent: a CTA that has finished a block of rows takes over the next CTA of the
// grid that has not been started (cluster launch control), so that setting up a CTA (barriers, tensor
// memory, tensor maps: about 2500 cycles), the first copies of the next block and the last stores of this one
// overlap, and the hardware still deals the blocks out as SMs become free, longest loops first.  One block
// to a CTA spent half of its 18,600 cycles outside the loop at 1024 tokens and 64 dimensions.
// Counters of turns and stages therefore run on over the blocks, and so do the barriers' phases: turn n of a
// ring of R uses stage n % R in the phase of tc_parity(n, R).
struct Block { int at, h, b; };         // first row, head, sequence
__device__ __forceinline__ Block block_of(long long w, int heads, int columns, int blocks, int rows, bool last_first) {
  const unsigned u = (unsigned)w, c = u % (unsigned)columns, k = u / (unsigned)columns;         // w: below 2^31, like any grid
  return Block{(last_first ? blocks - 1 - (int)k : (int)k) * rows, (int)(c % (unsigned)heads), (int)(c / (unsigned)heads)};
}

// ---- forward ------------------------------------------------------------------------------------
// One CTA per 256 queries of a head: two tiles of 128 that share every key and value tile, so that while
// one tile's four warps are at their exponentials the other's products run.
//   warps 0-3, 4-7   softmax of query tile 0, 1     warp 8  bulk copies     warps 9, 10  products of tile 0, 1
// (one warp for the products of both spent half its time in waits while the tensor cores ran dry: a warp can
// queue little ahead of them)
// Tensor memory: scores S_t at 128 t; head dimensions up to 64: O_t at 256 + 64 t and P_t apart at
// 384 + 64 t, so that S of the next key tile is computed while P of this one is formed; above 64: O_t at
// 256 + 128 t and P_t over S_t.
// The maximum that the exponents refer to is only raised when it has grown by more than 2^8 (P then
// stays below 256, and the sum and O below that times the length): rescaling O is rare.
// Measured: 16 x 1024, 12 heads of 64, causal: 58 us (446 TFLOP/s), bound by the softmax warps: a pair of 128 x 128
// tiles takes them some 3800 cycles, of which the exponentials alone need 2048.  2 x 4096, 16 heads of 128 over 4,
// ragged: 265 us (811 TFLOP/s), where S, softmax and P V of a tile follow one another because P lies over S.
constexpr int kFwdThreads = 384;       // three warpgroups: 168 registers a thread at launch, 64,512 in all
template <int NP> struct Fwd {
  static constexpr uint32_t tile = kT * 128 * NP;
  static constexpr int q_ring = NP == 1 ? 2 : 1, ring = NP == 1 ? 3 : 2;              // pairs of Q tiles; stages of K and of V
  static constexpr uint32_t k = 2 * q_ring * tile, v = k + ring * tile, bars = v + ring * tile;
  static constexpr size_t smem = bars + 320;
  static constexpr uint32_t o = 256, p = NP == 1 ? 384 : 0, o_step = NP == 1 ? 64 : 128, p_step = NP == 1 ? 64 : 128;
};
template <int NP> struct FwdBars {
  TcQueue queue;
  uint64_t q_full[Fwd<NP>::q_ring], q_empty[Fwd<NP>::q_ring], k_full[Fwd<NP>::ring], k_empty[Fwd<NP>::ring], v_full[Fwd<NP>::ring],
      v_empty[Fwd<NP>::ring], s_full[2], s_free[2], p_ready[2], pv_done[2], o_free[2], turn[2], finished[2];
  uint32_t tmem;
};

template <int NP>
__global__ void __launch_bounds__(kFwdThreads, 1)
attn_forward(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
             const __grid_constant__ CUtensorMap mv, const Sizes z, int blocks, const View o, float *__restrict__ lse) {
  typedef Fwd<NP> F;
  extern __shared__ __align__(1024) uint8_t base[];         // all of the CTA's shared memory: starts on a 1024-byte boundary
  static_assert(sizeof(FwdBars<NP>) <= 320, "barriers behind the tiles");
  FwdBars<NP> &bar = *reinterpret_cast<FwdBars<NP> *>(base + F::bars);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t sq = smem_u32(base), sk = sq + F::k, sv = sq + F::v;

  if (threadIdx.x == 0) {
    tc_queue_init(bar.queue, 11);
    for (int i = 0; i < F::q_ring; ++i) { mbar_init(smem_u32(&bar.q_full[i]), 1); mbar_init(smem_u32(&bar.q_empty[i]), 8); }
    for (int i = 0; i < F::ring; ++i) {
      mbar_init(smem_u32(&bar.k_full[i]), 1); mbar_init(smem_u32(&bar.k_empty[i]), 2);
      mbar_init(smem_u32(&bar.v_full[i]), 1); mbar_init(smem_u32(&bar.v_empty[i]), 2);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&bar.s_full[t]), 1); mbar_init(smem_u32(&bar.s_free[t]), 4);
      mbar_init(smem_u32(&bar.p_ready[t]), 4); mbar_init(smem_u32(&bar.pv_done[t]), 1);
      mbar_init(smem_u32(&bar.o_free[t]), 4); mbar_init(smem_u32(&bar.turn[t]), 4);
      mbar_init(smem_u32(&bar.finished[t]), 1);
    }
    mbar_init_fence();
  }
  if (warp == 9) tc_alloc(&bar.tmem, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = bar.tmem;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  long long deadline = clock64() + z.wait;       // of the waits for one block of rows
  const int columns = z.heads * z.batch;

  // the sequence's lengths and the key tiles that each query tile of a block sees
  struct Work { int lq, lk, n[2], tiles; };
  auto work_of = [&](const Block &w) {
    Work k;
    k.lq = used(z.q_lens, w.b, z.tq);
    k.lk = used(z.kv_lens, w.b, z.tk);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int first = w.at + t * kT, last = min(first + kT, k.lq) - 1;
      const int keys = first >= k.lq ? 0 : z.causal ? min(k.lk, last + k.lk - k.lq + 1) : k.lk;
      k.n[t] = keys > 0 ? (keys + kT - 1) / kT : 0;
    }
    k.tiles = max(k.n[0], k.n[1]);
    return k;
  };
  auto block = [&](long long at) { return block_of(at, z.heads, columns, blocks, 2 * kT, z.causal); };

  if (warp >= 8) {
    tc_regs_down<56>();            // 128 x 56 + 256 x 224 = 64,512
    if (warp == 8) {
      if (tc_elect()) {
        bool ok = true;
        int qn = 0, kn = 0, vn = 0;        // blocks and tiles issued
        int seq = 0, asked = 0;
        for (long long at = blockIdx.x; at >= 0 && ok; at = tc_queue_next_one(bar.queue, seq++, deadline, ok)) {
          deadline = clock64() + z.wait;
          if (!(ok = tc_queue_ask(bar.queue, seq, deadline))) break;
          ++asked;
          const Block w = block(at);
          const Work k = work_of(w);
          if (k.tiles == 0) continue;
          const int hk = w.h / z.group;
          if (!(ok = tc_wait_released(bar.q_empty, qn, F::q_ring, deadline))) break;
          uint64_t *full = &bar.q_full[qn % F::q_ring];
          const uint32_t q = sq + qn % F::q_ring * 2 * F::tile;
          mbar_expect_tx(smem_u32(full), 2 * F::tile);
          load_tile<NP>(q, &mq, w.at, w.h, batch_of(z, kQ, w.b), smem_u32(full));
          load_tile<NP>(q + F::tile, &mq, w.at + kT, w.h, batch_of(z, kQ, w.b), smem_u32(full));
          ++qn;
          for (int j = 0; j <= k.tiles; ++j) {         // K runs one tile ahead of V
            if (j < k.tiles) {
              if (!(ok = tc_wait_released(bar.k_empty, kn, F::ring, deadline))) break;
              full = &bar.k_full[kn % F::ring];
              mbar_expect_tx(smem_u32(full), F::tile);
              load_tile<NP>(sk + kn % F::ring * F::tile, &mk, j * kT, hk, batch_of(z, kK, w.b), smem_u32(full));
              ++kn;
            }
            if (j > 0) {
              if (!(ok = tc_wait_released(bar.v_empty, vn, F::ring, deadline))) break;
              full = &bar.v_full[vn % F::ring];
              mbar_expect_tx(smem_u32(full), F::tile);
              load_tile<NP>(sv + vn % F::ring * F::tile, &mv, (j - 1) * kT, hk, batch_of(z, kV, w.b), smem_u32(full));
              ++vn;
            }
          }
        }
        if (!ok) atomicOr(z.status, CDG_ST_TIMEOUT);
        tc_drain(bar.queue.full, asked, 2);
        tc_drain(bar.q_full, qn, F::q_ring);
        tc_drain(bar.k_full, kn, F::ring);
        tc_drain(bar.v_full, vn, F::ring);
      }
    } else if (warp < 11) {
      const int t = warp - 9;
      const uint32_t s_at = tm + t * kT;
      bool ok = true;
      int qn = 0, kn = 0, vn = 0, sn = 0, pn = 0, on = 0;      // blocks, tiles of K and V, products S_t and P_t V, blocks with any
      int seq = 0;
      for (long long at = blockIdx.x; at >= 0 && ok; at = tc_queue_next(bar.queue, seq++, deadline, ok)) {
        deadline = clock64() + z.wait;
        const Block w = block(at);
        const Work k = work_of(w);
        if (k.tiles == 0) continue;
        const int mine = t == 0 ? k.n[0] : k.n[1];
        const uint32_t q_tile = sq + (qn % F::q_ring * 2 + t) * F::tile;
        // S_t of key tile j; the stage of K is released when both tiles have used it (or have no use for it)
        auto scores = [&](int j) {
          const int ks = kn % F::ring;
          if (!tc_wait(&bar.k_full[ks], tc_parity(kn, F::ring), deadline)) return false;
          ++kn;
          // up to 64 head dimensions: the one before is in registers; above, P_t lies over it, and its product is over
          if (j < mine && sn > 0 && !tc_wait(NP == 1 ? &bar.s_free[t] : &bar.pv_done[t], (sn - 1) & 1, deadline)) return false;
          tc_fence_after();
          if (tc_elect()) {
            if (j < mine) {
              mma_scores<NP>(s_at, q_tile, sk + ks * F::tile);
              tc_commit(&bar.s_full[t]);
            }
            tc_commit(&bar.k_empty[ks]);
          }
          __syncwarp();
          sn += j < mine;
          return true;
        };
        if (!(ok = tc_wait(&bar.q_full[qn % F::q_ring], tc_parity(qn, F::q_ring), deadline) && scores(0))) break;
        for (int j = 0; j < k.tiles; ++j) {
          const int vs = vn % F::ring;
          if (NP == 1 && j + 1 < k.tiles && !(ok = scores(j + 1))) break;
          if (!(ok = tc_wait(&bar.v_full[vs], tc_parity(vn, F::ring), deadline))) break;
          ++vn;
          // (both warps zero the rows past the sequence, each before its own product)
          if (z.kv_lens && (j + 1) * kT > k.lk) zero_rows<NP>(base + F::v + vs * F::tile, k.lk - j * kT);
          if (j < mine) {
            if (j == 0 && on > 0 && !(ok = tc_wait(&bar.o_free[t], (on - 1) & 1, deadline))) break;
            if (!(ok = tc_wait(&bar.p_ready[t], pn & 1, deadline))) break;
            ++pn;
          }
          tc_fence_after();
          if (tc_elect()) {
            if (j < mine) {
              mma_rows<NP>(tm + F::o + t * F::o_step, tm + F::p + t * F::p_step, 32, sv + vs * F::tile, j > 0);
              tc_commit(&bar.pv_done[t]);
            }
            tc_commit(&bar.v_empty[vs]);
          }
          __syncwarp();
          if (NP == 2 && j + 1 < k.tiles && !(ok = scores(j + 1))) break;
        }
        ++qn;
        on += mine > 0;
      }
      if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
      tc_finish(&bar.finished[t]);
    }
  } else {
    tc_regs_up<224>();
    const int t = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tm + lanes + t * kT, tp = tm + lanes + F::p + t * F::p_step, to = tm + lanes + F::o + t * F::o_step;
    const float a = z.a;
    bool ok = true;
    int qn = 0, sn = 0, gn = 0;          // blocks, score tiles of this half, and turns of both halves
    int seq = 0;
    for (long long at = blockIdx.x; at >= 0 && ok; at = tc_queue_next(bar.queue, seq++, deadline, ok)) {
      deadline = clock64() + z.wait;
      const Block w = block(at);
      const Work k = work_of(w);
      const int mine = t == 0 ? k.n[0] : k.n[1], i = w.at + t * kT + row;
      const int keys = i >= k.lq ? 0 : z.causal ? min(k.lk, i + k.lk - k.lq + 1) : k.lk;     // this row sees keys 0 .. keys - 1
      float ref = -INFINITY, sum = 0.0f;
      for (int j = 0; j < k.tiles; ++j, ++gn) {
        // Above 64 head dimensions the two halves take turns at the exponentials, so that one's fall into the
        // other's products (2 x 4096, 16/4 heads of 128, ragged: 300 -> 273 us; at 64 dimensions the exponentials
        // are the longer part and turns cost 58 -> 62 us).  A half that does not see the tile passes its turn on,
        // so that both count the same turns.
        auto my_turn = [&]() { return t == 0 ? gn == 0 || tc_wait(&bar.turn[1], (gn - 1) & 1, deadline) : tc_wait(&bar.turn[0], gn & 1, deadline); };
        if (j >= mine) {
          if (NP == 1) break;
          if (!(ok = my_turn())) break;
          tc_warp_arrive(&bar.turn[t]);
          continue;
        }
        if (!(ok = tc_wait(&bar.s_full[t], sn & 1, deadline))) break;
        tc_fence_after();
        uint32_t v[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tc_load32(ts + c * 32, v[c]);
        tc_wait_ld();
        if (NP == 1) {
          tc_fence_before();
          tc_warp_arrive(&bar.s_free[t]);
        }
        if (z.negative) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 32; ++e) v[c][e] ^= 0x80000000u;
        }
        const int left = keys - j * kT;
        if (__any_sync(0xffffffffu, left < kT)) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (c * 32 + e >= left) v[c][e] = 0xff800000u;
        }
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int e = 0; e < 32; ++e)
#pragma unroll
          for (int c = 0; c < 4; ++c) top[c] = fmaxf(top[c], __uint_as_float(v[c][e]));
        const float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        // raise the reference where the maximum has outgrown it by 2^8, or where there was none
        const bool raise = mx > ref && (ref == -INFINITY || (mx - ref) * a > 8.0f);
        const float factor = raise ? exp2_fast((ref - mx) * a) : 1.0f;
        if (raise) { ref = mx; sum *= factor; }
        const float shift = ref == -INFINITY ? 0.0f : -ref * a;
        if (j > 0 && __any_sync(0xffffffffu, raise)) {
          if (!(ok = tc_wait(&bar.pv_done[t], (sn - 1) & 1, deadline))) break;
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < 2 * NP; ++c) {
            uint32_t u[32];
            tc_load32(to + c * 32, u);
            tc_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) u[e] = __float_as_uint(__uint_as_float(u[e]) * factor);
            tc_store32(to + c * 32, u);
          }
        }
        if (NP == 2 && !(ok = my_turn())) break;
        float2 part[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
        uint32_t u[2][32];
#pragma unroll
        for (int e = 0; e < 128; e += 2) {
          const float2 x = fma2(make_float2(__uint_as_float(v[e >> 5][e & 31]), __uint_as_float(v[e >> 5][(e & 31) + 1])),
                                make_float2(a, a), make_float2(shift, shift));
          const float2 p = exp2_two(x);
          part[(e >> 1) & 1] = add2(part[(e >> 1) & 1], p);
          u[e >> 6][(e >> 1) & 31] = pack(p.x, p.y);
        }
        if (NP == 2) tc_warp_arrive(&bar.turn[t]);
        // P's place is free when its last product is over (above 64 head dimensions S came after that)
        if (NP == 1 && j > 0 && !(ok = tc_wait(&bar.pv_done[t], (sn - 1) & 1, deadline))) break;
        tc_fence_after();
        tc_store32(tp, u[0]);
        tc_store32(tp + 32, u[1]);
        sum += (part[0].x + part[0].y) + (part[1].x + part[1].y);
        tc_wait_st();
        tc_fence_before();
        tc_warp_arrive(&bar.p_ready[t]);
        ++sn;
      }
      if (!ok) break;
      bf16 *dst = o.p + (long long)w.b * o.b + (long long)w.h * o.h;
      if (mine > 0) {
        if (!(ok = tc_wait(&bar.pv_done[t], (sn - 1) & 1, deadline))) break;
        tc_fence_after();
        // the tile of Q is no longer read: it takes O on its way out
        uint8_t *tile = base + (qn % F::q_ring * 2 + t) * F::tile;
        const float inv = keys > 0 && sum > 0.0f ? 1.0f / sum : 0.0f;
        uint32_t u[2 * NP][16];
#pragma unroll
        for (int c = 0; c < 2 * NP; ++c) {
          uint32_t v[32];
          tc_load32(to + c * 32, v);
          tc_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; ++e) u[c][e] = keys > 0 ? pack(__uint_as_float(v[2 * e]) * inv, __uint_as_float(v[2 * e + 1]) * inv) : 0u;
        }
        tc_fence_before();
        tc_warp_arrive(&bar.o_free[t]);
#pragma unroll
        for (int c = 0; c < 2 * NP; ++c) stage_row<NP>(tile, row, c * 32, u[c]);
        __syncwarp();
        write_rows<NP>(tile, (warp & 3) * 32, 32, w.at + t * kT, z.tq, z, dst, o.t);
      } else {
        write_zeros<NP>((warp & 3) * 32, 32, w.at + t * kT, z.tq, z, dst, o.t);
      }
      if (i < z.tq)
        lse[((long long)w.b * z.heads + w.h) * z.tq + i] = keys > 0 ? fmaf(ref, a * kLn2, logf(sum)) : -INFINITY;
      if (k.tiles > 0) {
        tc_proxy_fence();                // the next copy into the tile comes after these reads
        tc_warp_arrive(&bar.q_empty[qn % F::q_ring]);
        ++qn;
      }
    }
    tc_wait_st();                        // (of a rescaled O, where a wait expired after it)
    if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) { tc_fence_after(); tc_free(tm, 512); }
}

// ---- backward -----------------------------------------------------------------------------------
// For every query row: -delta = -sum_d do o, and -lse in base 2 (-infinity where the row sees nothing, so
// that its recomputed probabilities are 0).  Rows are padded to whole tiles: [batch][heads][2][rows], first lse.
// Eight lanes to a row and head, 16 bytes a lane.
__global__ void __launch_bounds__(256) attn_delta(const Sizes z, const View d_o, const View o, const float *__restrict__ lse,
                                                  float *__restrict__ out, int padded) {
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const long long group = ((long long)blockIdx.x * 256 + threadIdx.x) >> 3;
  const int l = threadIdx.x & 7;
  const int h = (int)(group % z.heads), i = (int)(group / z.heads % padded), b = (int)(group / z.heads / padded);
  if (b >= z.batch) return;
  float s = 0.0f, l2 = -INFINITY;
  if (i < used(z.q_lens, b, z.tq)) {
    const bf16 *x = d_o.p + b * d_o.b + i * d_o.t + h * d_o.h, *y = o.p + b * o.b + i * o.t + h * o.h;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      if (c * 64 + l * 8 >= z.dim) continue;
      const uint4 u = *reinterpret_cast<const uint4 *>(x + c * 64 + l * 8), w = *reinterpret_cast<const uint4 *>(y + c * 64 + l * 8);
      const uint32_t ua[4] = {u.x, u.y, u.z, u.w}, wa[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&ua[e]));
        const float2 g = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&wa[e]));
        s = fmaf(f.x, g.x, fmaf(f.y, g.y, s));
      }
    }
    l2 = lse[((long long)b * z.heads + h) * z.tq + i] * -kLog2e;
    if (l2 == INFINITY) l2 = -INFINITY;
  }
#pragma unroll
  for (int off = 4; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off, 8);
  if (l == 0) {
    float *row = out + ((long long)b * z.heads + h) * 2 * padded + i;
    row[0] = l2;
    row[padded] = l2 == -INFINITY ? 0.0f : -s;
  }
}

// 512 bytes of a row of `out` above; both addresses are multiples of 16 bytes
__device__ __forceinline__ void load_line(uint32_t dst, const float *src, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(kT * 4), "r"(bar) : "memory");
}

// Both backward kernels: eight warps work on a tile of scores, four on its columns 0..63 and four on
// 64..127, one row per thread.
//   warps 0-7  P and dS     warp 8  bulk copies     warp 9  S and dP     warp 10  the products with P and dS
//   warps 12-15  the results of a block, on their way out while the next block's scores are worked on (with
//                warps 0-7 doing it a block of 5 tiles spent 4800 of its 15,600 cycles there: 98 -> 86 us each)
// (two warps issue products because one can queue little ahead of the tensor cores and spends some 200 cycles
// between two products in its waits)
// What a warp reports as ready, or is told is done, has a barrier for even and one for odd turns: a warp may be
// a turn ahead of another, and with one barrier it would complete a phase in the other's place.
// Measured, 16 x 1024, 12 heads of 64, causal: dk and dv 85 us, dq 87 us.  A tile takes 2050 cycles, of which the
// exponentials need 1024; the rest is dS and the way of S, dP, P and dS to and from tensor memory.  Letting the
// two halves take turns at the exponentials is no faster, since a warp by itself does only one in 14 cycles.
// The rings are as deep as shared memory allows: a tile of Q (or K) is used twice, at the beginning and at
// the end of its turn, and a copy takes about 1700 cycles; with two stages each the products waited for it
// (3500 cycles a tile at 128 head dimensions).
//
// Where there are few tiles of rows, the loop over the other axis is dealt out over a cluster of CTAs, whose
// fp32 sums are joined through distributed shared memory, in the order of their ranks.
// fp32 sums of a tile in shared memory, [128][DP] with 16-byte pieces permuted by row, so that neither a row
// per thread nor a row per warp meets bank conflicts
template <int NP> __device__ __forceinline__ uint32_t sum_at(int row, int piece) {
  return (uint32_t)(row * NP * 256 + (((piece & ~7) | ((piece ^ row) & 7)) << 4));
}
template <int NP>
__device__ __forceinline__ void keep_sums(uint8_t *sums, int row, int c0, const uint32_t (&w)[32]) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    *reinterpret_cast<uint4 *>(sums + sum_at<NP>(row, (c0 >> 2) + i)) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}
// this CTA's share of the rows of a tile: the cluster's sums added up, scaled and written
template <int NP>
__device__ __forceinline__ void join_sums(uint32_t sums, int ranks, int rank, int thread, int threads, int token0, int tokens, int used_tokens,
                                          const Sizes &z, float f, bf16 *dst, long long stride) {
  const int rows = kT / ranks, per = z.dim >> 3;
  for (int i = thread; i < rows * per; i += threads) {
    const int r = rank * rows + i / per, chunk = i % per, token = token0 + r;
    if (token >= tokens) continue;
    float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f), b = a;
    if (token < used_tokens)
      for (int k = 0; k < ranks; ++k) {
        const float4 u = tc_peer_load(sums + sum_at<NP>(r, 2 * chunk), k), v = tc_peer_load(sums + sum_at<NP>(r, 2 * chunk + 1), k);
        a.x += u.x; a.y += u.y; a.z += u.z; a.w += u.w;
        b.x += v.x; b.y += v.y; b.z += v.z; b.w += v.w;
      }
    *reinterpret_cast<uint4 *>(dst + (long long)token * stride + chunk * 8) =
        make_uint4(pack(a.x * f, a.y * f), pack(a.z * f, a.w * f), pack(b.x * f, b.y * f), pack(b.z * f, b.w * f));
  }
}

// dk and dv of 128 keys: the loop runs over the query tiles of every query head that reads this key head.
// Scores are transposed (a row is a key), so that P^T and dS^T are the row operands of
//   dv += P^T dO,  dk += dS^T Q,    with  S^T = K Q^T,  dP^T = V dO^T.
// Summing over query tiles and heads in a fixed order makes the result the same bits every time.
// Tensor memory holds dv and dk and regions of 128 columns for the scores.  In turn n region n & 1 holds S, then,
// over each half's own scores, P and dS.  Up to 64 head dimensions dP has a third region, so that S of the next
// turn is computed while this one's P is formed.  Above, dP takes the region that S of this turn does not lie
// in; once it is in registers, S of the next turn is computed in its place while dS is being formed, and dP of
// the next turn follows when both products of this one are over.
constexpr int kBwdThreads = 512;       // 128 registers a thread at launch: 128 x 56 + 128 x 88 + 256 x 184 after they are moved
template <int NP> struct Dkv {
  static constexpr uint32_t tile = kT * 128 * NP;
  static constexpr int kv_ring = NP == 1 ? 2 : 1, q_ring = NP == 1 ? 4 : 3, do_ring = NP == 1 ? 3 : 2, line_ring = NP == 1 ? 4 : 2;
  static constexpr uint32_t line = 2 * kT * 4;              // lse and delta of a query tile
  static constexpr uint32_t q = 2 * kv_ring * tile, d_o = q + q_ring * tile, lines = d_o + do_ring * tile, bars = lines + line_ring * line;
  static constexpr size_t smem = bars + 448;
  static constexpr uint32_t dv = 512 - 128 * NP, dk = dv + 64 * NP;
};
template <int NP> struct DkvBars {
  TcQueue queue;
  uint64_t kv_full[Dkv<NP>::kv_ring], kv_empty[Dkv<NP>::kv_ring], q_full[Dkv<NP>::q_ring], q_empty[Dkv<NP>::q_ring], do_full[Dkv<NP>::do_ring],
      do_empty[Dkv<NP>::do_ring], line_full[Dkv<NP>::line_ring], line_empty[Dkv<NP>::line_ring], s_full[2], dp_full, dp_free,
      p_ready[2], ds_ready[2], done[2], block_done, acc_free, finished[2];       // [2]: even and odd turns
  uint32_t tmem;
};

template <int NP>
__global__ void __launch_bounds__(kBwdThreads, 1)
attn_backward_kv(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                 const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo, const Sizes z, int blocks,
                 const float *__restrict__ lines, int padded, const View dk, const View dv) {
  typedef Dkv<NP> F;
  extern __shared__ __align__(1024) uint8_t base[];
  static_assert(sizeof(DkvBars<NP>) <= 448, "barriers behind the tiles");
  DkvBars<NP> &bar = *reinterpret_cast<DkvBars<NP> *>(base + F::bars);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t s0 = smem_u32(base), sq = s0 + F::q, sdo = s0 + F::d_o;
  float *sline = reinterpret_cast<float *>(base + F::lines);      // [ring][2][128]
  const int ranks = (int)tc_cluster_size(), rank = (int)tc_cluster_rank(), kv_heads = z.heads / z.group;

  if (threadIdx.x == 0) {
    tc_queue_init(bar.queue, 15);
    for (int i = 0; i < F::kv_ring; ++i) { mbar_init(smem_u32(&bar.kv_full[i]), 1); mbar_init(smem_u32(&bar.kv_empty[i]), 4); }
    for (int i = 0; i < F::q_ring; ++i) { mbar_init(smem_u32(&bar.q_full[i]), 1); mbar_init(smem_u32(&bar.q_empty[i]), 1); }
    for (int i = 0; i < F::do_ring; ++i) { mbar_init(smem_u32(&bar.do_full[i]), 1); mbar_init(smem_u32(&bar.do_empty[i]), 2); }
    for (int i = 0; i < F::line_ring; ++i) { mbar_init(smem_u32(&bar.line_full[i]), 1); mbar_init(smem_u32(&bar.line_empty[i]), 8); }
    for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&bar.s_full[i]), 1); mbar_init(smem_u32(&bar.done[i]), 1); }
    mbar_init(smem_u32(&bar.dp_full), 1); mbar_init(smem_u32(&bar.dp_free), 8);
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&bar.p_ready[i]), 8); mbar_init(smem_u32(&bar.ds_ready[i]), 8);
      mbar_init(smem_u32(&bar.finished[i]), 1);
    }
    mbar_init(smem_u32(&bar.block_done), 1); mbar_init(smem_u32(&bar.acc_free), 4);
    mbar_init_fence();
  }
  if (warp == 9) tc_alloc(&bar.tmem, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = bar.tmem;
  const auto dp_at = [](int n) { return NP == 1 ? 256u : (uint32_t)(~n & 1) * kT; };
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  long long deadline = clock64() + z.wait;       // of the waits for one block of rows
  const int columns = kv_heads * z.batch;

  // query tiles first .. first + per - 1 see a key of the block; over the heads of the group this CTA takes
  // numbers rank, rank + ranks, ... of per * group, `total` of them
  struct Work { int lq, lk, first, per, total; };
  auto work_of = [&](const Block &w) {
    Work k;
    k.lq = used(z.q_lens, w.b, z.tq);
    k.lk = used(z.kv_lens, w.b, z.tk);
    k.first = w.at >= k.lk ? 0 : z.causal ? max(0, w.at - (k.lk - k.lq)) / kT : 0;
    k.per = w.at >= k.lk ? 0 : max(0, (k.lq + kT - 1) / kT - k.first);
    k.total = (k.per * z.group - rank + ranks - 1) / ranks;
    return k;
  };
  // where the loop stands: query tile first + tile of head `head` of the group
  struct Turn { int head, tile; };
  auto step = [&](Turn &t, const Work &k, int by) {
    for (t.tile += by; t.tile >= k.per; t.tile -= k.per) ++t.head;
  };
  auto start = [&](const Work &k) {
    Turn t = {0, 0};
    if (k.total > 0) step(t, k, rank);
    return t;
  };
  auto query0 = [&](const Work &k, const Turn &t) { return (k.first + t.tile) * kT; };
  // the first keys are seen by the most queries; a cluster takes one block and asks for no more
  auto block = [&](long long at) { return block_of(at, kv_heads, columns, blocks, kT, false); };
  const long long mine0 = blockIdx.x / ranks;

  if (warp >= 8 && warp < 12) {
    tc_regs_down<56>();
    if (warp == 8) {
      if (tc_elect()) {
        bool ok = true;
        int cn = 0, qn = 0, dn = 0, ln = 0;
        int seq = 0, asked = 0;
        for (long long at = mine0; at >= 0 && ok; at = ranks > 1 ? -1 : tc_queue_next_one(bar.queue, seq++, deadline, ok)) {
          deadline = clock64() + z.wait;
          if (ranks == 1) {
            if (!(ok = tc_queue_ask(bar.queue, seq, deadline))) break;
            ++asked;
          }
          const Block w = block(at);
          const Work k = work_of(w);
          if (k.total == 0) continue;
          if (!(ok = tc_wait_released(bar.kv_empty, cn, F::kv_ring, deadline))) break;
          uint64_t *full = &bar.kv_full[cn % F::kv_ring];
          const uint32_t kv = s0 + cn % F::kv_ring * 2 * F::tile;
          mbar_expect_tx(smem_u32(full), 2 * F::tile);
          load_tile<NP>(kv, &mk, w.at, w.h, batch_of(z, kK, w.b), smem_u32(full));
          load_tile<NP>(kv + F::tile, &mv, w.at, w.h, batch_of(z, kV, w.b), smem_u32(full));
          ++cn;
          Turn t = start(k);
          for (int it = 0; it < k.total; ++it, step(t, k, ranks)) {
            const int h = w.h * z.group + t.head, i0 = query0(k, t);
            if (!(ok = tc_wait_released(bar.q_empty, qn, F::q_ring, deadline))) break;
            full = &bar.q_full[qn % F::q_ring];
            mbar_expect_tx(smem_u32(full), F::tile);
            load_tile<NP>(sq + qn % F::q_ring * F::tile, &mq, i0, h, batch_of(z, kQ, w.b), smem_u32(full));
            ++qn;
            if (!(ok = tc_wait_released(bar.line_empty, ln, F::line_ring, deadline))) break;
            full = &bar.line_full[ln % F::line_ring];
            const float *line = lines + ((long long)w.b * z.heads + h) * 2 * padded + i0;
            float *to = sline + ln % F::line_ring * 2 * kT;
            mbar_expect_tx(smem_u32(full), F::line);
            load_line(smem_u32(to), line, smem_u32(full));
            load_line(smem_u32(to + kT), line + padded, smem_u32(full));
            ++ln;
            if (!(ok = tc_wait_released(bar.do_empty, dn, F::do_ring, deadline))) break;
            full = &bar.do_full[dn % F::do_ring];
            mbar_expect_tx(smem_u32(full), F::tile);
            load_tile<NP>(sdo + dn % F::do_ring * F::tile, &mdo, i0, h, batch_of(z, kDo, w.b), smem_u32(full));
            ++dn;
          }
        }
        if (!ok) atomicOr(z.status, CDG_ST_TIMEOUT);
        tc_drain(bar.queue.full, asked, 2);
        tc_drain(bar.kv_full, cn, F::kv_ring);
        tc_drain(bar.q_full, qn, F::q_ring);
        tc_drain(bar.line_full, ln, F::line_ring);
        tc_drain(bar.do_full, dn, F::do_ring);
      }
    } else if (warp <= 10) {
      bool ok = true;
      int cn = 0, n = 0;                   // blocks and turns
      int seq = 0;
      for (long long at = mine0; at >= 0 && ok; at = ranks > 1 ? -1 : tc_queue_next(bar.queue, seq++, deadline, ok)) {
        deadline = clock64() + z.wait;
        const Block w = block(at);
        const Work k = work_of(w);
        if (k.total == 0) continue;
        // a tile has landed; its rows past the sequence's queries are zeroed (by either warp, each before its own product)
        auto arrived = [&](uint64_t *full, uint32_t tiles, int ring, const Turn &t, int m) {
          const int s = m % ring, left = k.lq - query0(k, t);
          if (!tc_wait(&full[s], tc_parity(m, ring), deadline)) return false;
          if (z.q_lens && left < kT) zero_rows<NP>(base + tiles + s * F::tile, left);
          return true;
        };
        const uint32_t sk = s0 + cn % F::kv_ring * 2 * F::tile, sv = sk + F::tile;
        if (warp == 9) {
          if (!(ok = tc_wait(&bar.kv_full[cn % F::kv_ring], tc_parity(cn, F::kv_ring), deadline))) break;
          // S of turn `t`, number m: its region was last used by the products of turn m - 2, or by dP of turn m - 1
          auto scores = [&](const Turn &t, int m) {
            if (!arrived(bar.q_full, F::q, F::q_ring, t, m)) return false;
            if (NP == 1 ? m > 1 && !tc_wait(&bar.done[m & 1], tc_parity(m - 2, 2), deadline)
                        : m > 0 && !tc_wait(&bar.dp_free, (m - 1) & 1, deadline)) return false;
            tc_fence_after();
            if (tc_elect()) {
              mma_scores<NP>(tm + (m & 1) * kT, sk, sq + m % F::q_ring * F::tile);
              tc_commit(&bar.s_full[m & 1]);
            }
            __syncwarp();
            return true;
          };
          Turn t = start(k);
          ok = scores(t, n);
          for (int it = 0; it < k.total && ok; ++it, ++n) {
            if (!(ok = arrived(bar.do_full, F::d_o, F::do_ring, t, n))) break;
            if (n > 0 && !(ok = NP == 1 ? tc_wait(&bar.dp_free, (n - 1) & 1, deadline)
                                        : tc_wait(&bar.done[(n - 1) & 1], tc_parity(n - 1, 2), deadline))) break;
            tc_fence_after();
            if (tc_elect()) {
              mma_scores<NP>(tm + dp_at(n), sv, sdo + n % F::do_ring * F::tile);
              tc_commit(&bar.dp_full);
              tc_commit(&bar.do_empty[n % F::do_ring]);
            }
            __syncwarp();
            step(t, k, ranks);
            ok = it + 1 == k.total || scores(t, n + 1);
          }
          if (!ok) break;
        } else {
          Turn t = start(k);
          for (int it = 0; it < k.total; ++it, ++n, step(t, k, ranks)) {
            const uint32_t here = tm + (n & 1) * kT;
            if (it == 0 && cn > 0 && !(ok = tc_wait(&bar.acc_free, (cn - 1) & 1, deadline))) break;
            if (!(ok = arrived(bar.do_full, F::d_o, F::do_ring, t, n) && tc_wait(&bar.p_ready[n & 1], tc_parity(n, 2), deadline))) break;
            tc_fence_after();
            if (tc_elect()) {
              mma_rows<NP>(tm + F::dv, here, 64, sdo + n % F::do_ring * F::tile, it > 0);
              tc_commit(&bar.do_empty[n % F::do_ring]);
            }
            __syncwarp();
            if (!(ok = tc_wait(&bar.ds_ready[n & 1], tc_parity(n, 2), deadline))) break;
            tc_fence_after();
            if (tc_elect()) {
              mma_rows<NP>(tm + F::dk, here + 32, 64, sq + n % F::q_ring * F::tile, it > 0);
              tc_commit(&bar.done[n & 1]);
              if (it + 1 == k.total) tc_commit(&bar.block_done);
              tc_commit(&bar.q_empty[n % F::q_ring]);
            }
            __syncwarp();
          }
        }
        ++cn;
      }
      if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
      tc_finish(&bar.finished[warp - 9]);
    }
  } else if (warp >= 12) {
    tc_regs_down<88>();
    const int row = (warp & 3) * 32 + lane;
    const uint32_t lanes = tm + ((uint32_t)((warp & 3) * 32) << 16);
    bool ok = true;
    int cn = 0;
    int seq = 0;
    for (long long at = mine0; at >= 0 && ok; at = ranks > 1 ? -1 : tc_queue_next(bar.queue, seq++, deadline, ok)) {
      deadline = clock64() + z.wait;
      const Block w = block(at);
      const Work k = work_of(w);
      const int j = w.at + row;
      // through shared memory that no product reads any more
      if (k.total > 0 && !(ok = tc_wait(&bar.block_done, cn & 1, deadline))) break;
      tc_fence_after();
#pragma unroll 1
      for (int which = 0; which < 2; ++which) {
        const View &out = which ? dk : dv;
        const float f = which ? z.scale : 1.0f;
        bf16 *dst = out.p + (long long)w.b * out.b + (long long)w.h * out.h;
        if (ranks == 1 && k.total == 0) {
          write_zeros<NP>((warp & 3) * 32, 32, w.at, z.tk, z, dst, out.t);
          continue;
        }
        uint8_t *tile = base + (ranks > 1 ? which * 2 : cn % F::kv_ring * 2 + which) * F::tile;
#pragma unroll
        for (int c = 0; c < 2 * NP; ++c) {
          uint32_t v[32] = {}, u[16];
          if (k.total > 0) {
            tc_load32(lanes + (which ? F::dk : F::dv) + c * 32, v);
            tc_wait_ld();
          }
          if (ranks > 1) {
            keep_sums<NP>(tile, row, c * 32, v);
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) u[e] = j < k.lk ? pack(__uint_as_float(v[2 * e]) * f, __uint_as_float(v[2 * e + 1]) * f) : 0u;
            stage_row<NP>(tile, row, c * 32, u);
          }
        }
      }
      if (ranks == 1 && k.total > 0) {
        tc_fence_before();
        tc_warp_arrive(&bar.acc_free);
        for (int which = 0; which < 2; ++which) {
          const View &out = which ? dk : dv;
          write_rows<NP>(base + (cn % F::kv_ring * 2 + which) * F::tile, (warp & 3) * 32, 32, w.at, z.tk, z,
                         out.p + (long long)w.b * out.b + (long long)w.h * out.h, out.t);
        }
        tc_proxy_fence();              // the next copy into the tiles comes after these reads
        tc_warp_arrive(&bar.kv_empty[cn % F::kv_ring]);
        ++cn;
      }
    }
    if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
  } else {
    tc_regs_up<184>();
    const int half = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = tm + ((uint32_t)((warp & 3) * 32) << 16), mine = lanes + half * 64;
    const float a = z.negative ? -z.a : z.a;
    const float2 aa = make_float2(a, a);
    bool ok = true;
    int n = 0;
    int seq = 0;
    for (long long at = mine0; at >= 0 && ok; at = ranks > 1 ? -1 : tc_queue_next(bar.queue, seq++, deadline, ok)) {
      deadline = clock64() + z.wait;
      const Block w = block(at);
      const Work k = work_of(w);
      const int j = w.at + row, off = k.lk - k.lq;
      Turn t = start(k);
      for (int it = 0; it < k.total; ++it, ++n, step(t, k, ranks)) {
        const int ls = n % F::line_ring, i0 = query0(k, t) + half * 64;
        const uint32_t here = mine + (n & 1) * kT, there = mine + dp_at(n);
        const float *l2 = sline + ls * 2 * kT + half * 64, *delta = l2 + kT;
        if (!(ok = tc_wait(&bar.line_full[ls], tc_parity(n, F::line_ring), deadline))) break;
        if (!(ok = tc_wait(&bar.s_full[n & 1], tc_parity(n, 2), deadline))) break;
        tc_fence_after();
        uint32_t v[2][32], u[32];
        tc_load32(here, v[0]);
        tc_load32(here + 32, v[1]);
        tc_wait_ld();
        float p[64];
#pragma unroll
        for (int e = 0; e < 64; e += 4) {
          const float4 l = *reinterpret_cast<const float4 *>(l2 + e);
          const float2 x = exp2_two(fma2(two(v, e), aa, make_float2(l.x, l.y))), y = exp2_two(fma2(two(v, e + 2), aa, make_float2(l.z, l.w)));
          p[e] = x.x; p[e + 1] = x.y; p[e + 2] = y.x; p[e + 3] = y.y;
        }
        // under the causal rule key j is seen by queries from j - off on
        const int from = z.causal ? j - off - i0 : 0;
        if (__any_sync(0xffffffffu, from > 0)) {
#pragma unroll
          for (int e = 0; e < 64; ++e)
            if (e < from) p[e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) u[e] = pack(p[2 * e], p[2 * e + 1]);
        tc_store32(here, u);
        tc_wait_st();
        tc_fence_before();
        tc_warp_arrive(&bar.p_ready[n & 1]);
        if (!(ok = tc_wait(&bar.dp_full, n & 1, deadline))) break;
        tc_fence_after();
        tc_load32(there, v[0]);
        tc_load32(there + 32, v[1]);
        tc_wait_ld();
        tc_fence_before();
        tc_warp_arrive(&bar.dp_free);
#pragma unroll
        for (int e = 0; e < 64; e += 4) {
          const float4 d = *reinterpret_cast<const float4 *>(delta + e);
          const float2 x = mul2(make_float2(p[e], p[e + 1]), add2(two(v, e), make_float2(d.x, d.y)));
          const float2 y = mul2(make_float2(p[e + 2], p[e + 3]), add2(two(v, e + 2), make_float2(d.z, d.w)));
          u[e / 2] = pack(x.x, x.y);
          u[e / 2 + 1] = pack(y.x, y.y);
        }
        tc_store32(here + 32, u);
        tc_wait_st();
        tc_fence_before();
        tc_warp_arrive(&bar.ds_ready[n & 1]);
        if (lane == 0) mbar_arrive(smem_u32(&bar.line_empty[ls]));
      }
    }
    if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) { tc_fence_after(); tc_free(tm, 512); }
  if (ranks > 1) {             // one block to a cluster
    tc_cluster_sync();
    if (warp < 8) {
      const int half = warp >> 2;
      const View &out = half ? dk : dv;
      const Block w = block_of(blockIdx.x / ranks, kv_heads, columns, blocks, kT, false);
      join_sums<NP>(s0 + half * 2 * F::tile, ranks, rank, threadIdx.x & 127, 128, w.at, z.tk, used(z.kv_lens, w.b, z.tk), z,
                    half ? z.scale : 1.0f, out.p + (long long)w.b * out.b + (long long)w.h * out.h, out.t);
    }
    tc_cluster_sync();            // no CTA leaves while another reads its sums
  }
}

// dq of 128 queries of a head: dq += dS K over the key tiles it sees, S = Q K^T, dP = dO V^T.  A pass of its
// own: adding dq's parts up from the kernel above would need additions to memory in no fixed order.
// Tensor memory: S at 0, dP at 128, dq at 256, dS in turn at 384 and 448 (so that one is being read by the product).
// The exponentials of one key tile are formed together with dS of the one before, so that the special
// function units work while the FMA units do.
template <int NP> struct Dq {
  static constexpr uint32_t tile = kT * 128 * NP;
  static constexpr int q_ring = NP == 1 ? 2 : 1, k_ring = NP == 1 ? 5 : 3, v_ring = NP == 1 ? 3 : 2;       // q: Q and dO
  static constexpr uint32_t k = 2 * q_ring * tile, v = k + k_ring * tile, bars = v + v_ring * tile;
  static constexpr size_t smem = bars + 384;
  static constexpr uint32_t dq = 256, ds = 384;
};
template <int NP> struct DqBars {
  TcQueue queue;
  uint64_t q_full[Dq<NP>::q_ring], q_empty[Dq<NP>::q_ring], k_full[Dq<NP>::k_ring], k_empty[Dq<NP>::k_ring], v_full[Dq<NP>::v_ring],
      v_empty[Dq<NP>::v_ring], s_full, s_free, dp_full, dp_free, ds_ready[2], dq_done[2], block_done, acc_free, finished[2];       // [2]: even and odd turns
  uint32_t tmem;
};

template <int NP>
__global__ void __launch_bounds__(kBwdThreads, 1)
attn_backward_q(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo, const Sizes z, int blocks,
                const float *__restrict__ lines, int padded, const View dq) {
  typedef Dq<NP> F;
  extern __shared__ __align__(1024) uint8_t base[];
  static_assert(sizeof(DqBars<NP>) <= 384, "barriers behind the tiles");
  DqBars<NP> &bar = *reinterpret_cast<DqBars<NP> *>(base + F::bars);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t s0 = smem_u32(base), sk = s0 + F::k, sv = s0 + F::v;
  const int ranks = (int)tc_cluster_size(), rank = (int)tc_cluster_rank();

  if (threadIdx.x == 0) {
    tc_queue_init(bar.queue, 15);
    for (int i = 0; i < F::q_ring; ++i) { mbar_init(smem_u32(&bar.q_full[i]), 1); mbar_init(smem_u32(&bar.q_empty[i]), 4); }
    for (int i = 0; i < F::k_ring; ++i) { mbar_init(smem_u32(&bar.k_full[i]), 1); mbar_init(smem_u32(&bar.k_empty[i]), 1); }
    for (int i = 0; i < F::v_ring; ++i) { mbar_init(smem_u32(&bar.v_full[i]), 1); mbar_init(smem_u32(&bar.v_empty[i]), 1); }
    mbar_init(smem_u32(&bar.s_full), 1); mbar_init(smem_u32(&bar.dp_full), 1);
    mbar_init(smem_u32(&bar.s_free), 8); mbar_init(smem_u32(&bar.dp_free), 8);
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&bar.ds_ready[i]), 8); mbar_init(smem_u32(&bar.dq_done[i]), 1);
      mbar_init(smem_u32(&bar.finished[i]), 1);
    }
    mbar_init(smem_u32(&bar.block_done), 1); mbar_init(smem_u32(&bar.acc_free), 4);
    mbar_init_fence();
  }
  if (warp == 9) tc_alloc(&bar.tmem, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = bar.tmem;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  long long deadline = clock64() + z.wait;       // of the waits for one block of rows
  const int columns = z.heads * z.batch;

  // key tiles rank, rank + ranks, ... of those that the block sees, `total` of them
  struct Work { int lq, lk, total; };
  auto work_of = [&](const Block &w) {
    Work k;
    k.lq = used(z.q_lens, w.b, z.tq);
    k.lk = used(z.kv_lens, w.b, z.tk);
    const int seen = w.at >= k.lq ? 0 : z.causal ? min(k.lk, min(w.at + kT, k.lq) + k.lk - k.lq) : k.lk;
    k.total = ((seen > 0 ? (seen + kT - 1) / kT : 0) - rank + ranks - 1) / ranks;
    return k;
  };
  auto block = [&](long long at) { return block_of(at, z.heads, columns, blocks, kT, z.causal); };
  const long long mine0 = blockIdx.x / ranks;

  if (warp >= 8 && warp < 12) {
    tc_regs_down<56>();
    if (warp == 8) {
      if (tc_elect()) {
        bool ok = true;
        int qn = 0, kn = 0, vn = 0;
        int seq = 0, asked = 0;
        for (long long at = mine0; at >= 0 && ok; at = ranks > 1 ? -1 : tc_queue_next_one(bar.queue, seq++, deadline, ok)) {
          deadline = clock64() + z.wait;
          if (ranks == 1) {
            if (!(ok = tc_queue_ask(bar.queue, seq, deadline))) break;
            ++asked;
          }
          const Block w = block(at);
          const Work k = work_of(w);
          if (k.total == 0) continue;
          const int hk = w.h / z.group;
          if (!(ok = tc_wait_released(bar.q_empty, qn, F::q_ring, deadline))) break;
          uint64_t *full = &bar.q_full[qn % F::q_ring];
          const uint32_t q = s0 + qn % F::q_ring * 2 * F::tile;
          mbar_expect_tx(smem_u32(full), 2 * F::tile);
          load_tile<NP>(q, &mq, w.at, w.h, batch_of(z, kQ, w.b), smem_u32(full));
          load_tile<NP>(q + F::tile, &mdo, w.at, w.h, batch_of(z, kDo, w.b), smem_u32(full));
          ++qn;
          for (int it = 0; it < k.total; ++it) {
            const int j0 = (rank + it * ranks) * kT;
            if (!(ok = tc_wait_released(bar.k_empty, kn, F::k_ring, deadline))) break;
            full = &bar.k_full[kn % F::k_ring];
            mbar_expect_tx(smem_u32(full), F::tile);
            load_tile<NP>(sk + kn % F::k_ring * F::tile, &mk, j0, hk, batch_of(z, kK, w.b), smem_u32(full));
            ++kn;
            if (!(ok = tc_wait_released(bar.v_empty, vn, F::v_ring, deadline))) break;
            full = &bar.v_full[vn % F::v_ring];
            mbar_expect_tx(smem_u32(full), F::tile);
            load_tile<NP>(sv + vn % F::v_ring * F::tile, &mv, j0, hk, batch_of(z, kV, w.b), smem_u32(full));
            ++vn;
          }
        }
        if (!ok) atomicOr(z.status, CDG_ST_TIMEOUT);
        tc_drain(bar.queue.full, asked, 2);
        tc_drain(bar.q_full, qn, F::q_ring);
        tc_drain(bar.k_full, kn, F::k_ring);
        tc_drain(bar.v_full, vn, F::v_ring);
      }
    } else if (warp < 11) {
      bool ok = true;
      int qn = 0, n = 0;                 // blocks, and turns whose S (warp 9) or dq (warp 10) has been issued
      int seq = 0;
      for (long long at = mine0; at >= 0 && ok; at = ranks > 1 ? -1 : tc_queue_next(bar.queue, seq++, deadline, ok)) {
        deadline = clock64() + z.wait;
        const Block w = block(at);
        const Work k = work_of(w);
        if (k.total == 0) continue;
        const uint32_t q = s0 + qn % F::q_ring * 2 * F::tile;
        if (warp == 9) {
          auto scores = [&](int it) {    // S of tile it: K has landed, its rows past the sequence are zeroed, the S before is in registers
            const int s = n % F::k_ring, left = k.lk - (rank + it * ranks) * kT;
            if (!tc_wait(&bar.k_full[s], tc_parity(n, F::k_ring), deadline)) return false;
            if (z.kv_lens && left < kT) zero_rows<NP>(base + F::k + s * F::tile, left);
            if (n > 0 && !tc_wait(&bar.s_free, (n - 1) & 1, deadline)) return false;
            tc_fence_after();
            if (tc_elect()) {
              mma_scores<NP>(tm, q, sk + s * F::tile);
              tc_commit(&bar.s_full);
            }
            __syncwarp();
            ++n;
            return true;
          };
          auto gradients = [&](int m) {  // dP of turn m likewise
            const int s = m % F::v_ring;
            if (!tc_wait(&bar.v_full[s], tc_parity(m, F::v_ring), deadline) || (m > 0 && !tc_wait(&bar.dp_free, (m - 1) & 1, deadline))) return false;
            tc_fence_after();
            if (tc_elect()) {
              mma_scores<NP>(tm + kT, q + F::tile, sv + s * F::tile);
              tc_commit(&bar.dp_full);
              tc_commit(&bar.v_empty[s]);
            }
            __syncwarp();
            return true;
          };
          ok = tc_wait(&bar.q_full[qn % F::q_ring], tc_parity(qn, F::q_ring), deadline) && scores(0);
          for (int it = 0; it < k.total && ok; ++it) ok = gradients(n - 1) && (it + 1 == k.total || scores(it + 1));
          if (!ok) break;
        } else {
          for (int it = 0; it < k.total; ++it, ++n) {
            const int ks = n % F::k_ring;
            if (it == 0 && qn > 0 && !(ok = tc_wait(&bar.acc_free, (qn - 1) & 1, deadline))) break;
            if (!(ok = tc_wait(&bar.ds_ready[n & 1], tc_parity(n, 2), deadline))) break;
            tc_fence_after();
            if (tc_elect()) {
              mma_rows<NP>(tm + F::dq, tm + F::ds + (n & 1) * 64, 32, sk + ks * F::tile, it > 0);
              tc_commit(&bar.dq_done[n & 1]);
              if (it + 1 == k.total) tc_commit(&bar.block_done);
              tc_commit(&bar.k_empty[ks]);
            }
            __syncwarp();
          }
        }
        ++qn;
      }
      if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
      tc_finish(&bar.finished[warp - 9]);
    }
  } else if (warp >= 12) {
    tc_regs_down<88>();
    const int row = (warp & 3) * 32 + lane;
    const uint32_t lanes = tm + ((uint32_t)((warp & 3) * 32) << 16);
    bool ok = true;
    int qn = 0;
    int seq = 0;
    for (long long at = mine0; at >= 0 && ok; at = ranks > 1 ? -1 : tc_queue_next(bar.queue, seq++, deadline, ok)) {
      deadline = clock64() + z.wait;
      const Block w = block(at);
      const Work k = work_of(w);
      const int i = w.at + row;
      const bool sees = i < k.lq && (z.causal ? i + k.lk - k.lq + 1 : k.lk) > 0;
      bf16 *dst = dq.p + (long long)w.b * dq.b + (long long)w.h * dq.h;
      if (ranks == 1 && k.total == 0) {
        write_zeros<NP>((warp & 3) * 32, 32, w.at, z.tq, z, dst, dq.t);
        continue;
      }
      // through the tile of Q, which no product reads any more
      if (k.total > 0 && !(ok = tc_wait(&bar.block_done, qn & 1, deadline))) break;
      tc_fence_after();
      uint8_t *tile = base + (ranks > 1 ? 0 : qn % F::q_ring * 2) * F::tile;
#pragma unroll
      for (int c = 0; c < 2 * NP; ++c) {
        uint32_t v[32] = {}, u[16];
        if (k.total > 0) {
          tc_load32(lanes + F::dq + c * 32, v);
          tc_wait_ld();
        }
        if (ranks > 1) {
          keep_sums<NP>(tile, row, c * 32, v);
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) u[e] = sees ? pack(__uint_as_float(v[2 * e]) * z.scale, __uint_as_float(v[2 * e + 1]) * z.scale) : 0u;
          stage_row<NP>(tile, row, c * 32, u);
        }
      }
      if (ranks == 1) {
        tc_fence_before();
        tc_warp_arrive(&bar.acc_free);
        write_rows<NP>(tile, (warp & 3) * 32, 32, w.at, z.tq, z, dst, dq.t);
        tc_proxy_fence();              // the next copy into the tile comes after these reads
        tc_warp_arrive(&bar.q_empty[qn % F::q_ring]);
        ++qn;
      }
    }
    if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
  } else {
    tc_regs_up<184>();
    const int half = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = tm + ((uint32_t)((warp & 3) * 32) << 16), ts = lanes + half * 64, tdp = ts + kT;
    const float a = z.negative ? -z.a : z.a;
    const float2 aa = make_float2(a, a);
    bool ok = true;
    int n = 0;
    int seq = 0;
    for (long long at = mine0; at >= 0 && ok; at = ranks > 1 ? -1 : tc_queue_next(bar.queue, seq++, deadline, ok)) {
      deadline = clock64() + z.wait;
      const Block w = block(at);
      const Work k = work_of(w);
      const int i = w.at + row, keys = i >= k.lq ? 0 : z.causal ? min(k.lk, i + k.lk - k.lq + 1) : k.lk;
      float2 ll = make_float2(-INFINITY, -INFINITY), dd = make_float2(0.0f, 0.0f);          // -lse, -delta
      if (i < padded) {
        const float *line = lines + ((long long)w.b * z.heads + w.h) * 2 * padded + i;
        ll.x = ll.y = line[0];
        dd.x = dd.y = line[padded];
      }
      float p[64];
      if (k.total > 0) {
        if (!(ok = tc_wait(&bar.s_full, n & 1, deadline))) break;
        tc_fence_after();
        uint32_t v[2][32];
        tc_load32(ts, v[0]);
        tc_load32(ts + 32, v[1]);
        tc_wait_ld();
        tc_fence_before();
        tc_warp_arrive(&bar.s_free);
#pragma unroll
        for (int e = 0; e < 64; e += 2) {
          const float2 y = fma2(two(v, e), aa, ll), x = exp2_two(y);
          p[e] = x.x;
          p[e + 1] = x.y;
        }
      }
      for (int it = 0; it < k.total; ++it, ++n) {
        const bool next = it + 1 < k.total;
        if (!(ok = (!next || tc_wait(&bar.s_full, (n + 1) & 1, deadline)) && tc_wait(&bar.dp_full, n & 1, deadline))) break;
        tc_fence_after();
        uint32_t v[32] = {}, u[2][32], x[32];
        tc_load32(tdp, u[0]);
        tc_load32(tdp + 32, u[1]);
        if (next) tc_load32(ts, v);
        tc_wait_ld();
        tc_fence_before();
        tc_warp_arrive(&bar.dp_free);
        const int left = keys - (rank + it * ranks) * kT - half * 64;
        if (__any_sync(0xffffffffu, left < 64)) {       // replaces P and dP: whatever lies there is not used
#pragma unroll
          for (int e = 0; e < 64; ++e)
            if (e >= left) { p[e] = 0.0f; u[e >> 5][e & 31] = 0u; }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          if (c == 1) {                // S's other half, when there are registers for it
            if (next) tc_load32(ts + 32, v);
            tc_wait_ld();
            tc_fence_before();
            if (next) tc_warp_arrive(&bar.s_free);
          }
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const int f = c * 32 + e;
            const float2 d = mul2(make_float2(p[f], p[f + 1]), add2(two(u, f), dd));
            x[f / 2] = pack(d.x, d.y);
            const float2 t = exp2_two(fma2(make_float2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), aa, ll));
            p[f] = t.x;
            p[f + 1] = t.y;
          }
        }
        if (n > 1) {               // the place of dS is free when its last product is over
          if (!(ok = tc_wait(&bar.dq_done[n & 1], tc_parity(n - 2, 2), deadline))) break;
          tc_fence_after();
        }
        tc_store32(lanes + F::ds + (n & 1) * 64 + half * 32, x);
        tc_wait_st();
        tc_fence_before();
        tc_warp_arrive(&bar.ds_ready[n & 1]);
      }
    }
    if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) { tc_fence_after(); tc_free(tm, 512); }
  if (ranks > 1) {             // one block to a cluster
    tc_cluster_sync();
    if (warp < 8) {
      const Block w = block_of(blockIdx.x / ranks, z.heads, columns, blocks, kT, z.causal);
      join_sums<NP>(s0, ranks, rank, threadIdx.x, 256, w.at, z.tq, used(z.q_lens, w.b, z.tq), z, z.scale,
                    dq.p + (long long)w.b * dq.b + (long long)w.h * dq.h, dq.t);
    }
    tc_cluster_sync();
  }
}

// ---- host ---------------------------------------------------------------------------------------
constexpr long long kMaxStride = 1ll << 38;   // elements; a tensor map holds byte strides below 2^40

bool in_ok(const long long s[3], int tokens, int heads, int dim) { return cdg_heads_in_ok(s, tokens, heads, dim, kMaxStride); }
bool out_ok(const long long s[3], int batch, int tokens, int heads, int dim) {
  return cdg_heads_out_ok(s, batch, tokens, heads, dim, kMaxStride);
}

constexpr int kMaxTokens = 1 << 22;

bool shape_ok(const cdgrab_attention_shape *s) {
  if (!s || s->batch < 0 || s->batch > 65535 || s->len_q < 0 || s->len_kv < 0 || s->heads < 1 || s->kv_heads < 1 ||
      s->heads > 65535 || s->heads % s->kv_heads != 0)
    return false;
  if (s->head_dim < 8 || s->head_dim > 128 || s->head_dim % 8 != 0 || (s->causal != 0 && s->causal != 1)) return false;
  // the grid's axes: batch x heads x CTAs of a cluster (up to 8), and tiles of tokens
  if ((long long)s->batch * s->heads > 0x0fffffffll || s->len_q > kMaxTokens || s->len_kv > kMaxTokens) return false;
  return isfinite(s->scale);
}

Sizes sizes_of(const cdgrab_attention_shape *s, const int32_t *q_lens, const int32_t *kv_lens, int *status) {
  // a wait may span a block's whole loop: the limit grows with loops of more than 65,536 tiles (a tile takes 2000 to 3800
  // cycles, the default limit allows 61,000)
  const double tiles = fmax((double)((s->len_q + kT - 1) / kT) * (s->heads / s->kv_heads), (double)((s->len_kv + kT - 1) / kT));
  const long long wait = (long long)((double)cdg_ops_wait_limit() * fmax(1.0, tiles / 65536));
  const int shared = (s->q_stride[0] > 0 ? 0 : kQ) | (s->k_stride[0] > 0 ? 0 : kK) | (s->v_stride[0] > 0 ? 0 : kV) |
                     (s->do_stride[0] > 0 ? 0 : kDo);
  return Sizes{s->batch, s->len_q, s->len_kv, s->heads, s->heads / s->kv_heads, s->head_dim, s->causal, s->scale,
               fmaxf(fabsf(s->scale) * kLog2e, 1e-30f), s->scale < 0.0f, shared, q_lens, kv_lens,
               wait, status};
}
View view(const void *p, const long long s[3]) { return View{(bf16 *)const_cast<void *>(p), s[0], s[1], s[2]}; }

// [batch][head][token][dim] as the copies see it, boxes of 64 dimensions by 128 tokens
bool map_of(CUtensorMap *m, const void *p, const long long s[3], int batch, int tokens, int heads, int dim) {
  const long long dims[4] = {dim, tokens, heads, s[0] > 0 ? batch : 1};
  // an axis of length one (or shared by the batch, read at 0) still needs a stride the copy engine takes
  const long long strides[4] = {1, s[1] > 0 ? s[1] : 64, s[2] > 0 ? s[2] : 64, s[0] > 0 ? s[0] : 64};
  return tc_encode(m, true, p, 4, dims, strides, kT);
}
template <int NP>
int forward(const cdgrab_attention_shape *s, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const Sizes &z,
            const View &o, float *lse, cudaStream_t st) {
  static CdgPerDevice flags;
  if (!tc_raise_limit(flags, attn_forward<NP>, Fwd<NP>::smem)) return CDGRAB_ERR_CUDA;
  const int blocks = (s->len_q + 2 * kT - 1) / (2 * kT);
  const long long all = (long long)s->heads * s->batch * blocks;
  if (all > 0x7fffffffll) return CDGRAB_ERR_INVALID;
  return cdg_launch_rc(cdg_ops_launch(attn_forward<NP>, dim3((unsigned)all), kFwdThreads, Fwd<NP>::smem, st, mq, mk, mv,
                                      z, blocks, o, lse));
}

// CTAs that share the loop of one block of rows: the number for which the estimated time, in turns of a
// loop, is least.  `longest` and `mean` are the turns of the longest block and on average, `all` the number of
// blocks.  A cluster sets up and joins anew for each block, which costs some three turns and half a turn for
// each of its CTAs, a single CTA about two in all.  (us at 1, 2, 4 CTAs, causal: dk and dv of one sequence of 4096, 16
// query heads of 128 over 4: 244, 139, 185; of 3 x 357 queries on 257 keys, 6 heads of 80 over 2: 28, 22, 20, and 22
// at 8; dq: 111, 154, 271 and 12, 14, 25.)
int split_of(double longest, double mean, long long all, int sms) {
  int best = 1;
  double least = 0.0;
  for (int c = 1; c <= 8 && (c == 1 || longest / c >= 1.0); c *= 2) {
    const double rounds = ceil((double)all * c / sms);
    const double turns = fmax(longest / c, rounds * mean / c) + (c > 1 ? (3.0 + 0.5 * c) * rounds : 2.0);
    if (c == 1 || turns < least) { best = c; least = turns; }
  }
  return best;
}
template <int NP>
int backward(const cdgrab_attention_shape *s, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const CUtensorMap &mdo,
             const Sizes &z, const float *lines, int padded, const View &dq, const View &dk, const View &dv, int sms, cudaStream_t st) {
  static CdgPerDevice kf, qf;
  if (!tc_raise_limit(kf, attn_backward_kv<NP>, Dkv<NP>::smem) || !tc_raise_limit(qf, attn_backward_q<NP>, Dq<NP>::smem)) return CDGRAB_ERR_CUDA;
  int rc = CDGRAB_OK;
  const int qt = (s->len_q + kT - 1) / kT, kt = (s->len_kv + kT - 1) / kT;
  const double part = s->causal ? 0.5 : 1.0;
  if (kt > 0) {
    const long long all = (long long)kt * s->kv_heads * s->batch;
    const int c = split_of((double)qt * z.group, part * qt * z.group, all, sms);
    rc = tc_launch_cluster(attn_backward_kv<NP>, dim3((unsigned)(all * c)), c, kBwdThreads, Dkv<NP>::smem, st, mq, mk, mv, mdo, z, kt, lines, padded,
                        dk, dv);
  }
  if (rc == CDGRAB_OK && qt > 0) {
    const long long all = (long long)qt * s->heads * s->batch;
    const int c = split_of(kt, part * kt, all, sms);
    rc = tc_launch_cluster(attn_backward_q<NP>, dim3((unsigned)(all * c)), c, kBwdThreads, Dq<NP>::smem, st, mq, mk, mv, mdo, z, qt, lines, padded, dq);
  }
  return rc;
}

}  // namespace

extern "C" int cdgrab_attention_forward(const cdgrab_attention_shape *s, const void *q, const void *k, const void *v,
                                        const int32_t *q_lens, const int32_t *kv_lens, void *o, float *lse,
                                        void *stream) {
  if (!shape_ok(s)) return CDGRAB_ERR_INVALID;
  if (s->batch == 0 || s->len_q == 0) return CDGRAB_OK;
  if (!q || !o || !lse || (s->len_kv > 0 && (!k || !v))) return CDGRAB_ERR_INVALID;
  if (!cdg_aligned(q, 16) || !cdg_aligned(k, 16) || !cdg_aligned(v, 16) || !cdg_aligned(o, 16) || !cdg_aligned(lse, 4) ||
      !cdg_aligned(q_lens, 4) || !cdg_aligned(kv_lens, 4))
    return CDGRAB_ERR_INVALID;
  if (!in_ok(s->q_stride, s->len_q, s->heads, s->head_dim) || !in_ok(s->k_stride, s->len_kv, s->kv_heads, s->head_dim) ||
      !in_ok(s->v_stride, s->len_kv, s->kv_heads, s->head_dim) ||
      !out_ok(s->o_stride, s->batch, s->len_q, s->heads, s->head_dim))
    return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  const Sizes z = sizes_of(s, q_lens, kv_lens, dev->status);
  // with no keys at all the maps of k and v are never used; they describe q
  const int tk = s->len_kv > 0 ? s->len_kv : 1;
  CUtensorMap mq, mk, mv;
  if (!map_of(&mq, q, s->q_stride, s->batch, s->len_q, s->heads, s->head_dim) ||
      !map_of(&mk, s->len_kv > 0 ? k : q, s->k_stride, s->batch, tk, s->kv_heads, s->head_dim) ||
      !map_of(&mv, s->len_kv > 0 ? v : q, s->v_stride, s->batch, tk, s->kv_heads, s->head_dim))
    return CDGRAB_ERR_CUDA;
  const View ov = view(o, s->o_stride);
  return s->head_dim <= 64 ? forward<1>(s, mq, mk, mv, z, ov, lse, (cudaStream_t)stream)
                           : forward<2>(s, mq, mk, mv, z, ov, lse, (cudaStream_t)stream);
}

extern "C" long long cdgrab_attention_workspace_bytes(const cdgrab_attention_shape *s) {
  if (!shape_ok(s)) return -1;
  const long long rows = ((long long)s->len_q + kT - 1) / kT * kT;        // lse and delta, padded to whole tiles
  return (long long)s->batch * s->heads * rows * 2 * 4 + 16;
}

extern "C" int cdgrab_attention_backward(const cdgrab_attention_shape *s, const void *d_o, const void *q, const void *k,
                                         const void *v, const void *o, const float *lse, const int32_t *q_lens,
                                         const int32_t *kv_lens, void *dq, void *dk, void *dv, void *workspace,
                                         long long workspace_bytes, void *stream) {
  if (!shape_ok(s)) return CDGRAB_ERR_INVALID;
  if (s->batch == 0 || (s->len_q == 0 && s->len_kv == 0)) return CDGRAB_OK;
  if (s->len_q > 0 && (!q || !o || !d_o || !dq || !lse)) return CDGRAB_ERR_INVALID;
  if (s->len_kv > 0 && (!k || !v || !dk || !dv)) return CDGRAB_ERR_INVALID;
  const void *ptrs[] = {d_o, q, k, v, o, dq, dk, dv, workspace};
  for (const void *p : ptrs)
    if (!cdg_aligned(p, 16)) return CDGRAB_ERR_INVALID;
  if (!cdg_aligned(lse, 4) || !cdg_aligned(q_lens, 4) || !cdg_aligned(kv_lens, 4)) return CDGRAB_ERR_INVALID;
  const long long *qs[] = {s->q_stride, s->o_stride, s->do_stride}, *ks[] = {s->k_stride, s->v_stride};
  for (const long long *t : qs)
    if (!in_ok(t, s->len_q, s->heads, s->head_dim)) return CDGRAB_ERR_INVALID;
  for (const long long *t : ks)
    if (!in_ok(t, s->len_kv, s->kv_heads, s->head_dim)) return CDGRAB_ERR_INVALID;
  if (!out_ok(s->dq_stride, s->batch, s->len_q, s->heads, s->head_dim) ||
      !out_ok(s->dk_stride, s->batch, s->len_kv, s->kv_heads, s->head_dim) ||
      !out_ok(s->dv_stride, s->batch, s->len_kv, s->kv_heads, s->head_dim))
    return CDGRAB_ERR_INVALID;
  if (!workspace || workspace_bytes < cdgrab_attention_workspace_bytes(s)) return CDGRAB_ERR_INVALID;
  // the grids: a block to a tile of rows, up to eight CTAs to a block
  if ((long long)((s->len_q + kT - 1) / kT) * s->heads * s->batch > 0x0fffffffll ||
      (long long)((s->len_kv + kT - 1) / kT) * s->kv_heads * s->batch > 0x0fffffffll)
    return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const Sizes z = sizes_of(s, q_lens, kv_lens, dev->status);
  float *lines = (float *)workspace;
  const long long padded = ((long long)s->len_q + kT - 1) / kT * kT;
  if (s->len_q > 0) {
    const long long blocks = (s->batch * padded * s->heads * 8 + 255) / 256;       // four to a tile
    const int rc = cdg_launch_rc(cdg_ops_launch(attn_delta, dim3((unsigned)blocks), 256, 0, st, z, view(d_o, s->do_stride),
                                                view(o, s->o_stride), lse, lines, (int)padded));
    if (rc != CDGRAB_OK) return rc;
  }
  // a tensor without tokens is never read; its map describes one that is there
  const bool has_q = s->len_q > 0, has_k = s->len_kv > 0;
  const int tq = has_q ? s->len_q : 1, tk = has_k ? s->len_kv : 1;
  CUtensorMap mq, mk, mv, mdo;
  if (!map_of(&mq, has_q ? q : k, s->q_stride, s->batch, tq, s->heads, s->head_dim) ||
      !map_of(&mk, has_k ? k : q, s->k_stride, s->batch, tk, s->kv_heads, s->head_dim) ||
      !map_of(&mv, has_k ? v : q, s->v_stride, s->batch, tk, s->kv_heads, s->head_dim) ||
      !map_of(&mdo, has_q ? d_o : k, s->do_stride, s->batch, tq, s->heads, s->head_dim))
    return CDGRAB_ERR_CUDA;
  const View vdq = view(dq, s->dq_stride), vdk = view(dk, s->dk_stride), vdv = view(dv, s->dv_stride);
  return s->head_dim <= 64 ? backward<1>(s, mq, mk, mv, mdo, z, lines, (int)padded, vdq, vdk, vdv, dev->sms, st)
                           : backward<2>(s, mq, mk, mv, mdo, z, lines, (int)padded, vdq, vdk, vdv, dev->sms, st);
}
