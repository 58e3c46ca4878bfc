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
  int *status;
};
struct View { bf16 *p; long long b, t, h; };

enum { kQ = 1, kK = 2, kV = 4, kDo = 8 };
__device__ __forceinline__ int batch_of(const Sizes &z, int which, int b) { return z.shared & which ? 0 : b; }
__device__ __forceinline__ int used(const int *lens, int b, int most) { return lens ? min(max(lens[b], 0), most) : most; }
__device__ __forceinline__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// two fp32 operations to an instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nmov.b64 z, {%6, %7};\n"
      "fma.rn.f32x2 z, x, y, z;\nmov.b64 {%0, %1}, z;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n.reg .b64 x, y;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nadd.rn.f32x2 x, x, y;\nmov.b64 {%0, %1}, x;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n.reg .b64 x, y;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nmul.rn.f32x2 x, x, y;\nmov.b64 {%0, %1}, x;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
// 2^x for two values on the FMA units: x = n + f, |f| <= 1/2, a polynomial of degree 5 for 2^f (a weighted
// least-squares fit of its relative error, 1.6e-7 at most), and n added to the exponent.  Below -126 the
// result is about 1e-38 instead of 0.
__device__ __forceinline__ float2 exp2_pair(float2 x) {
  const float2 magic = make_float2(12582912.0f, 12582912.0f);      // 1.5 x 2^23: the sum's last bits are n
  x.x = fmaxf(x.x, -126.0f);
  x.y = fmaxf(x.y, -126.0f);
  const float2 t = add2(x, magic);
  const float2 f = fma2(add2(t, make_float2(-12582912.0f, -12582912.0f)), make_float2(-1.0f, -1.0f), x);
  float2 r = make_float2(0.0013276375830173492f, 0.0013276375830173492f);
  r = fma2(r, f, make_float2(0.009675533510744572f, 0.009675533510744572f));
  r = fma2(r, f, make_float2(0.05550713464617729f, 0.05550713464617729f));
  r = fma2(r, f, make_float2(0.24022120237350464f, 0.24022120237350464f));
  r = fma2(r, f, make_float2(0.6931469440460205f, 0.6931469440460205f));
  r = fma2(r, f, make_float2(1.0000001192092896f, 1.0000001192092896f));
  r.x = __uint_as_float(__float_as_uint(r.x) + (__float_as_uint(t.x) << 23));
  r.y = __uint_as_float(__float_as_uint(r.y) + (__float_as_uint(t.y) << 23));
  return r;
}
// The exponentials are spread over both kinds of units: the special function units do 16 a cycle and SM,
// which bounds a tile of 128 x 128 at 1024 cycles; every fourth pair goes to the FMA units instead.
template <bool FMA> __device__ __forceinline__ float2 exp2_two(float2 x) {
  if (FMA) return exp2_pair(x);
  return make_float2(exp2_fast(x.x), exp2_fast(x.y));
}
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
template <int NP>
__device__ __forceinline__ void write_rows(const uint8_t *tile, int row0, int token0, int tokens, const Sizes &z, bf16 *dst, long long stride) {
  const int lane = threadIdx.x & 31, per = NP * 8;
  for (int i = lane; i < 32 * per; i += 32) {
    const int r = row0 + i / per, chunk = i % per;
    if (token0 + r < tokens && chunk * 8 < z.dim)
      *reinterpret_cast<uint4 *>(dst + (long long)(token0 + r) * stride + chunk * 8) =
          *reinterpret_cast<const uint4 *>(tile + (chunk >> 3) * kT * 128 + r * 128 + (((chunk & 7) ^ (r & 7)) << 4));
  }
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
constexpr int kFwdThreads = 384;       // three warpgroups: 168 registers a thread at launch, 64,512 in all
template <int NP> struct Fwd {
  static constexpr uint32_t tile = kT * 128 * NP;
  static constexpr int ring = NP == 1 ? 3 : 2;              // stages of K and of V
  static constexpr size_t smem = 2 * tile + 2 * ring * tile + 1024;
  static constexpr uint32_t o = 256, p = NP == 1 ? 384 : 0, o_step = NP == 1 ? 64 : 128, p_step = NP == 1 ? 64 : 128;
};

template <int NP>
__global__ void __launch_bounds__(kFwdThreads, 1)
attn_forward(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
             const __grid_constant__ CUtensorMap mv, const Sizes z, const View o, float *__restrict__ lse) {
  typedef Fwd<NP> F;
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t q_full, k_full[F::ring], k_empty[F::ring], v_full[F::ring], v_empty[F::ring], s_full[2],
      s_free[2], p_ready[2], pv_done[2];
  __shared__ uint32_t tmem_slot;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t *base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
  const uint32_t sq = smem_u32(base), sk = sq + 2 * F::tile, sv = sk + F::ring * F::tile;
  const int h = blockIdx.x % z.heads, b = blockIdx.x / z.heads, hk = h / z.group;
  // the longest query blocks of a causal batch start first
  const int i0 = (z.causal ? (int)gridDim.y - 1 - (int)blockIdx.y : (int)blockIdx.y) * 2 * kT;

  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&q_full), 1);
    for (int i = 0; i < F::ring; ++i) {
      mbar_init(smem_u32(&k_full[i]), 1); mbar_init(smem_u32(&k_empty[i]), 2);
      mbar_init(smem_u32(&v_full[i]), 1); mbar_init(smem_u32(&v_empty[i]), 2);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&s_full[t]), 1); mbar_init(smem_u32(&s_free[t]), 4);
      mbar_init(smem_u32(&p_ready[t]), 4); mbar_init(smem_u32(&pv_done[t]), 1);
    }
    mbar_init_fence();
  }
  if (warp == 9) tc_alloc(&tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = tmem_slot;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const long long deadline = clock64() + kCdgWaitCycles;

  const int lq = used(z.q_lens, b, z.tq), lk = used(z.kv_lens, b, z.tk);
  int n[2];                      // key tiles that query tile t sees
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int first = i0 + t * kT, last = min(first + kT, lq) - 1;
    const int keys = first >= lq ? 0 : z.causal ? min(lk, last + lk - lq + 1) : lk;
    n[t] = keys > 0 ? (keys + kT - 1) / kT : 0;
  }
  const int tiles = max(n[0], n[1]);

  if (warp >= 8) {
  tc_regs_down<56>();            // 128 x 56 + 256 x 224 = 64,512
  if (warp == 8) {
    if (tc_elect() && tiles > 0) {
      bool ok = true;
      int kn = 0, vn = 0;        // tiles issued
      mbar_expect_tx(smem_u32(&q_full), 2 * F::tile);
      load_tile<NP>(sq, &mq, i0, h, batch_of(z, kQ, b), smem_u32(&q_full));
      load_tile<NP>(sq + F::tile, &mq, i0 + kT, h, batch_of(z, kQ, b), smem_u32(&q_full));
      for (int j = 0; j <= tiles && ok; ++j) {         // K runs one tile ahead of V
        if (j < tiles) {
          const int s = j % F::ring;
          if (j >= F::ring) ok = mbar_wait(smem_u32(&k_empty[s]), (j / F::ring - 1) & 1, deadline);
          if (!ok) break;
          mbar_expect_tx(smem_u32(&k_full[s]), F::tile);
          load_tile<NP>(sk + s * F::tile, &mk, j * kT, hk, batch_of(z, kK, b), smem_u32(&k_full[s]));
          ++kn;
        }
        if (j > 0) {
          const int i = j - 1, s = i % F::ring;
          if (i >= F::ring) ok = mbar_wait(smem_u32(&v_empty[s]), (i / F::ring - 1) & 1, deadline);
          if (!ok) break;
          mbar_expect_tx(smem_u32(&v_full[s]), F::tile);
          load_tile<NP>(sv + s * F::tile, &mv, i * kT, hk, batch_of(z, kV, b), smem_u32(&v_full[s]));
          ++vn;
        }
      }
      if (!ok) {                 // let the copies in flight land before the CTA gives up its shared memory
        atomicOr(z.status, CDG_ST_TIMEOUT);
        mbar_wait(smem_u32(&q_full), 0, clock64() + kCdgWaitCycles);
        for (int i = max(0, kn - F::ring); i < kn; ++i) mbar_wait(smem_u32(&k_full[i % F::ring]), (i / F::ring) & 1, clock64() + kCdgWaitCycles);
        for (int i = max(0, vn - F::ring); i < vn; ++i) mbar_wait(smem_u32(&v_full[i % F::ring]), (i / F::ring) & 1, clock64() + kCdgWaitCycles);
      }
    }
  } else if (warp < 11) {
    const int t = warp - 9, mine = t == 0 ? n[0] : n[1];
    const uint32_t q_tile = sq + t * F::tile, s_at = tm + t * kT;
    // S_t of key tile j; the stage of K is released when both tiles have used it (or have no use for it)
    auto scores = [&](int j, uint64_t *before, uint32_t parity) {
      const int ks = j % F::ring;
      if (!tc_wait(&k_full[ks], (j / F::ring) & 1, deadline)) return false;
      if (j < mine && before && !tc_wait(before, parity, deadline)) return false;
      tc_fence_after();
      if (tc_elect()) {
        if (j < mine) {
          mma_scores<NP>(s_at, q_tile, sk + ks * F::tile);
          tc_commit(&s_full[t]);
        }
        tc_commit(&k_empty[ks]);
      }
      __syncwarp();
      return true;
    };
    bool ok = tiles == 0 || (tc_wait(&q_full, 0, deadline) && scores(0, nullptr, 0));
    for (int j = 0; j < tiles && ok; ++j) {
      const int vs = j % F::ring;
      // up to 64 head dimensions: S_t(j) is in registers, the next one may overwrite it
      if (NP == 1 && j + 1 < tiles && !(ok = scores(j + 1, &s_free[t], j & 1))) break;
      if (!(ok = tc_wait(&v_full[vs], (j / F::ring) & 1, deadline))) break;
      // (both warps zero the rows past the sequence, each before its own product)
      if (z.kv_lens && (j + 1) * kT > lk) zero_rows<NP>(base + 2 * F::tile + F::ring * F::tile + vs * F::tile, lk - j * kT);
      if (j < mine && !(ok = tc_wait(&p_ready[t], j & 1, deadline))) break;
      tc_fence_after();
      if (tc_elect()) {
        if (j < mine) {
          mma_rows<NP>(tm + F::o + t * F::o_step, tm + F::p + t * F::p_step, 32, sv + vs * F::tile, j > 0);
          tc_commit(&pv_done[t]);
        }
        tc_commit(&v_empty[vs]);
      }
      __syncwarp();
      // above: P_t lies over S_t, its product has to be over
      if (NP == 2 && j + 1 < tiles && !(ok = scores(j + 1, &pv_done[t], j & 1))) break;
    }
    if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
  }
  } else {
    tc_regs_up<224>();
    const int t = warp >> 2, row = (warp & 3) * 32 + lane, i = i0 + t * kT + row;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tm + lanes + t * kT, tp = tm + lanes + F::p + t * F::p_step, to = tm + lanes + F::o + t * F::o_step;
    const int keys = i >= lq ? 0 : z.causal ? min(lk, i + lk - lq + 1) : lk;     // this row sees keys 0 .. keys - 1
    const float a = z.a;
    float ref = -INFINITY, sum = 0.0f;
    bool ok = true;
    for (int j = 0; j < n[t]; ++j) {
      if (!(ok = tc_wait(&s_full[t], j & 1, deadline))) break;
      tc_fence_after();
      uint32_t v[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tc_load32(ts + c * 32, v[c]);
      tc_wait_ld();
      if (NP == 1) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_free[t]));
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
      if (j > 0 && !(ok = tc_wait(&pv_done[t], (j - 1) & 1, deadline))) break;
      if (j > 0 && __any_sync(0xffffffffu, raise)) {
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < 2 * NP; ++c) {
          uint32_t w[32];
          tc_load32(to + c * 32, w);
          tc_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) w[e] = __float_as_uint(__uint_as_float(w[e]) * factor);
          tc_store32(to + c * 32, w);
        }
      }
      float2 part[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
      for (int c = 0; c < 4; c += 2) {
        uint32_t w[32];
#pragma unroll
        for (int e = 0; e < 64; e += 2) {
          const float2 x = fma2(make_float2(__uint_as_float(v[c + (e >> 5)][e & 31]), __uint_as_float(v[c + (e >> 5)][(e & 31) + 1])),
                                make_float2(a, a), make_float2(shift, shift));
          const float2 p = (e & 6) == 0 ? exp2_two<true>(x) : exp2_two<false>(x);
          part[(e >> 1) & 1] = add2(part[(e >> 1) & 1], p);
          w[e >> 1] = pack(p.x, p.y);
        }
        tc_store32(tp + c * 16, w);
      }
      sum += (part[0].x + part[0].y) + (part[1].x + part[1].y);
      tc_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&p_ready[t]));
    }
    if (ok && n[t] > 0) ok = tc_wait(&pv_done[t], (n[t] - 1) & 1, deadline);
    if (ok && n[t] == 0 && tiles > 0) ok = tc_wait(&q_full, 0, deadline);     // its copy of Q has landed
    if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
    tc_fence_after();
    // the tile of Q is no longer read: it takes O on its way out
    uint8_t *tile = base + t * F::tile;
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int c = 0; c < 2 * NP; ++c) {
      uint32_t w[32], u[16];
      if (n[t] > 0) {
        tc_load32(to + c * 32, w);
        tc_wait_ld();
#pragma unroll
        for (int e = 0; e < 16; ++e)
          u[e] = keys > 0 ? pack(__uint_as_float(w[2 * e]) * inv, __uint_as_float(w[2 * e + 1]) * inv) : 0u;
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) u[e] = 0u;
      }
      stage_row<NP>(tile, row, c * 32, u);
    }
    __syncwarp();
    write_rows<NP>(tile, (warp & 3) * 32, i0 + t * kT, z.tq, z, o.p + (long long)b * o.b + (long long)h * o.h, o.t);
    if (i < z.tq)
      lse[((long long)b * z.heads + h) * z.tq + i] = keys > 0 ? fmaf(ref, a * kLn2, logf(sum)) : -INFINITY;
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
// (two warps issue products because one can queue little ahead of the tensor cores and spends some 200 cycles
// between two products in its waits)
// The rings are as deep as shared memory allows: a tile of Q (or K) is used twice, at the beginning and at
// the end of its turn, and a copy takes about 1700 cycles; with two stages each the products waited for it
// (3500 cycles a tile at 128 head dimensions).
constexpr int kBwdThreads = 352;

// Where there are few tiles of rows, the loop over the other axis is dealt out over a cluster of CTAs, whose
// fp32 sums are joined through distributed shared memory, in the order of their ranks.
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 peer_load(uint32_t addr, uint32_t rank) {
  uint32_t there;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(there) : "memory");
  return v;
}
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
        const float4 u = peer_load(sums + sum_at<NP>(r, 2 * chunk), k), v = peer_load(sums + sum_at<NP>(r, 2 * chunk + 1), k);
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
// Tensor memory: dv and dk from 256; the scores move between two regions of 128 columns.  In turn `it`
// region it & 1 holds S, then, over each half's own scores, P and dS; the other one holds dP.  Once dP is in
// registers, S of the next turn is computed in its place while dS is being formed; dP of the next turn
// follows when both products of this one are over.
template <int NP> struct Dkv {
  static constexpr uint32_t tile = kT * 128 * NP;
  static constexpr int q_ring = NP == 1 ? 4 : 3, do_ring = NP == 1 ? 4 : 2, line_ring = 2;
  static constexpr uint32_t line = 2 * kT * 4;              // lse and delta of a query tile
  static constexpr uint32_t lines = (2 + q_ring + do_ring) * tile, bars = lines + line_ring * line;
  static constexpr size_t smem = bars + 256;
  static constexpr uint32_t dv = 256, dk = 256 + 64 * NP;
};
template <int NP> struct DkvBars {
  uint64_t kv_full, q_full[Dkv<NP>::q_ring], q_empty[Dkv<NP>::q_ring], do_full[Dkv<NP>::do_ring], do_empty[Dkv<NP>::do_ring],
      line_full[Dkv<NP>::line_ring], line_empty[Dkv<NP>::line_ring], s_full, dp_full, dp_free, p_ready, ds_ready, done;
  uint32_t tmem;
};

template <int NP>
__global__ void __launch_bounds__(kBwdThreads, 1)
attn_backward_kv(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                 const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo, const Sizes z,
                 const float *__restrict__ lines, int padded, const View dk, const View dv) {
  typedef Dkv<NP> F;
  extern __shared__ __align__(1024) uint8_t base[];         // all of the CTA's shared memory: starts on a 1024-byte boundary
  static_assert(sizeof(DkvBars<NP>) <= 256, "barriers behind the tiles");
  DkvBars<NP> &bar = *reinterpret_cast<DkvBars<NP> *>(base + F::bars);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t sk = smem_u32(base), sv = sk + F::tile, sq = sv + F::tile, sdo = sq + F::q_ring * F::tile;
  float *sline = reinterpret_cast<float *>(base + F::lines);      // [ring][2][128]
  const int ranks = (int)cluster_size(), rank = (int)cluster_rank(), kv_heads = z.heads / z.group;
  const int column = blockIdx.x / ranks, hk = column % kv_heads, b = column / kv_heads;
  const int j0 = blockIdx.y * kT;            // the first keys, which most queries see, start first

  if (threadIdx.x == 0) {
    if (sk & 1023u) atomicOr(z.status, CDG_ST_TIMEOUT);      // (the copies' swizzle counts on it)
    mbar_init(smem_u32(&bar.kv_full), 1);
    for (int i = 0; i < F::q_ring; ++i) { mbar_init(smem_u32(&bar.q_full[i]), 1); mbar_init(smem_u32(&bar.q_empty[i]), 1); }
    for (int i = 0; i < F::do_ring; ++i) { mbar_init(smem_u32(&bar.do_full[i]), 1); mbar_init(smem_u32(&bar.do_empty[i]), 2); }
    for (int i = 0; i < F::line_ring; ++i) { mbar_init(smem_u32(&bar.line_full[i]), 1); mbar_init(smem_u32(&bar.line_empty[i]), 8); }
    mbar_init(smem_u32(&bar.s_full), 1); mbar_init(smem_u32(&bar.dp_full), 1);
    mbar_init(smem_u32(&bar.dp_free), 8); mbar_init(smem_u32(&bar.done), 1);
    mbar_init(smem_u32(&bar.p_ready), 8); mbar_init(smem_u32(&bar.ds_ready), 8);
    mbar_init_fence();
  }
  if (warp == 9) tc_alloc(&bar.tmem, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = bar.tmem;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const long long deadline = clock64() + kCdgWaitCycles;

  const int lq = used(z.q_lens, b, z.tq), lk = used(z.kv_lens, b, z.tk);
  // query tiles first .. last - 1 see key j0 or a later one of this tile
  const int first = j0 >= lk ? 0 : z.causal ? max(0, j0 - (lk - lq)) / kT : 0;
  const int last = j0 >= lk ? 0 : (lq + kT - 1) / kT;
  const int per = max(0, last - first), all = (sk & 1023u) ? 0 : per * z.group;
  const int total = (all - rank + ranks - 1) / ranks;        // this CTA's: numbers rank, rank + ranks, ...
  auto query0 = [&](int it) { return (first + (rank + it * ranks) % per) * kT; };

  if (warp == 8) {
    if (tc_elect() && total > 0) {
      bool ok = true;
      int qn = 0, dn = 0, ln = 0;
      mbar_expect_tx(smem_u32(&bar.kv_full), 2 * F::tile);
      load_tile<NP>(sk, &mk, j0, hk, batch_of(z, kK, b), smem_u32(&bar.kv_full));
      load_tile<NP>(sv, &mv, j0, hk, batch_of(z, kV, b), smem_u32(&bar.kv_full));
      for (int it = 0; it < total; ++it) {
        const int h = hk * z.group + (rank + it * ranks) / per, i0 = query0(it);
        const int qs = it % F::q_ring, os = it % F::do_ring, ls = it % F::line_ring;
        if (it >= F::q_ring && !(ok = mbar_wait(smem_u32(&bar.q_empty[qs]), (it / F::q_ring - 1) & 1, deadline))) break;
        mbar_expect_tx(smem_u32(&bar.q_full[qs]), F::tile);
        load_tile<NP>(sq + qs * F::tile, &mq, i0, h, batch_of(z, kQ, b), smem_u32(&bar.q_full[qs]));
        ++qn;
        if (it >= F::line_ring && !(ok = mbar_wait(smem_u32(&bar.line_empty[ls]), (it / F::line_ring - 1) & 1, deadline))) break;
        const float *line = lines + ((long long)b * z.heads + h) * 2 * padded + i0;
        mbar_expect_tx(smem_u32(&bar.line_full[ls]), F::line);
        load_line(smem_u32(sline + ls * 2 * kT), line, smem_u32(&bar.line_full[ls]));
        load_line(smem_u32(sline + ls * 2 * kT + kT), line + padded, smem_u32(&bar.line_full[ls]));
        ++ln;
        if (it >= F::do_ring && !(ok = mbar_wait(smem_u32(&bar.do_empty[os]), (it / F::do_ring - 1) & 1, deadline))) break;
        mbar_expect_tx(smem_u32(&bar.do_full[os]), F::tile);
        load_tile<NP>(sdo + os * F::tile, &mdo, i0, h, batch_of(z, kDo, b), smem_u32(&bar.do_full[os]));
        ++dn;
      }
      if (!ok) {
        atomicOr(z.status, CDG_ST_TIMEOUT);
        mbar_wait(smem_u32(&bar.kv_full), 0, clock64() + kCdgWaitCycles);
        for (int i = max(0, qn - F::q_ring); i < qn; ++i) mbar_wait(smem_u32(&bar.q_full[i % F::q_ring]), (i / F::q_ring) & 1, clock64() + kCdgWaitCycles);
        for (int i = max(0, ln - F::line_ring); i < ln; ++i) mbar_wait(smem_u32(&bar.line_full[i % F::line_ring]), (i / F::line_ring) & 1, clock64() + kCdgWaitCycles);
        for (int i = max(0, dn - F::do_ring); i < dn; ++i) mbar_wait(smem_u32(&bar.do_full[i % F::do_ring]), (i / F::do_ring) & 1, clock64() + kCdgWaitCycles);
      }
    }
  } else if (warp >= 9) {
    // (by either warp, each before its own product) a tile's rows past the sequence's queries are zeroed before any product reads them
    auto arrived = [&](uint64_t *full, uint32_t tiles, int ring, int it) {
      const int s = it % ring;
      if (!tc_wait(&full[s], (it / ring) & 1, deadline)) return false;
      const int left = lq - query0(it);
      if (z.q_lens && left < kT) zero_rows<NP>(base + (tiles - sk) + s * F::tile, left);
      return true;
    };
    bool ok = true;
    if (warp == 9) {
      auto scores = [&](int it) {
        if (!arrived(bar.q_full, sq, F::q_ring, it) || (it > 0 && !tc_wait(&bar.dp_free, (it - 1) & 1, deadline))) return false;
        tc_fence_after();
        if (tc_elect()) {
          mma_scores<NP>(tm + (it & 1) * kT, sk, sq + it % F::q_ring * F::tile);
          tc_commit(&bar.s_full);
        }
        __syncwarp();
        return true;
      };
      auto gradients = [&](int it) {
        if (!arrived(bar.do_full, sdo, F::do_ring, it) || (it > 0 && !tc_wait(&bar.done, (it - 1) & 1, deadline))) return false;
        tc_fence_after();
        if (tc_elect()) {
          mma_scores<NP>(tm + (~it & 1) * kT, sv, sdo + it % F::do_ring * F::tile);
          tc_commit(&bar.dp_full);
          tc_commit(&bar.do_empty[it % F::do_ring]);
        }
        __syncwarp();
        return true;
      };
      if (total > 0) ok = tc_wait(&bar.kv_full, 0, deadline);
      for (int it = 0; it < total && ok; ++it) ok = scores(it) && gradients(it);
    } else {
      for (int it = 0; it < total && ok; ++it) {
        const uint32_t here = tm + (it & 1) * kT;
        if (!(ok = arrived(bar.do_full, sdo, F::do_ring, it) && tc_wait(&bar.p_ready, it & 1, deadline))) break;
        tc_fence_after();
        if (tc_elect()) {
          mma_rows<NP>(tm + F::dv, here, 64, sdo + it % F::do_ring * F::tile, it > 0);
          tc_commit(&bar.do_empty[it % F::do_ring]);
        }
        __syncwarp();
        if (!(ok = tc_wait(&bar.ds_ready, it & 1, deadline))) break;
        tc_fence_after();
        if (tc_elect()) {
          mma_rows<NP>(tm + F::dk, here + 32, 64, sq + it % F::q_ring * F::tile, it > 0);
          tc_commit(&bar.done);
          tc_commit(&bar.q_empty[it % F::q_ring]);
        }
        __syncwarp();
      }
    }
    if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
  } else {
    const int half = warp >> 2, row = (warp & 3) * 32 + lane, j = j0 + row;
    const uint32_t mine = tm + ((uint32_t)((warp & 3) * 32) << 16) + half * 64;
    const float a = z.negative ? -z.a : z.a;
    const int off = lk - lq;
    bool ok = true;
    for (int it = 0; it < total; ++it) {
      const int ls = it % F::line_ring, i0 = query0(it) + half * 64;
      const uint32_t here = mine + (it & 1) * kT, there = mine + (~it & 1) * kT;
      const float *l2 = sline + ls * 2 * kT + half * 64, *delta = l2 + kT;
      if (!(ok = tc_wait(&bar.line_full[ls], (it / F::line_ring) & 1, deadline) && tc_wait(&bar.s_full, it & 1, deadline))) break;
      tc_fence_after();
      uint32_t v[2][32], w[32];
      tc_load32(here, v[0]);
      tc_load32(here + 32, v[1]);
      tc_wait_ld();
      float p[64];
#pragma unroll
      for (int e = 0; e < 64; e += 8) {
        const float4 l = *reinterpret_cast<const float4 *>(l2 + e), m = *reinterpret_cast<const float4 *>(l2 + e + 4);
        const float2 aa = make_float2(a, a);
        const float2 x0 = exp2_two<true>(fma2(two(v, e), aa, make_float2(l.x, l.y)));
        const float2 x1 = exp2_two<false>(fma2(two(v, e + 2), aa, make_float2(l.z, l.w)));
        const float2 x2 = exp2_two<false>(fma2(two(v, e + 4), aa, make_float2(m.x, m.y)));
        const float2 x3 = exp2_two<false>(fma2(two(v, e + 6), aa, make_float2(m.z, m.w)));
        p[e] = x0.x; p[e + 1] = x0.y; p[e + 2] = x1.x; p[e + 3] = x1.y;
        p[e + 4] = x2.x; p[e + 5] = x2.y; p[e + 6] = x3.x; p[e + 7] = x3.y;
      }
      // under the causal rule key j is seen by queries from j - off on
      const int from = z.causal ? j - off - i0 : 0;
      if (__any_sync(0xffffffffu, from > 0)) {
#pragma unroll
        for (int e = 0; e < 64; ++e)
          if (e < from) p[e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < 32; ++e) w[e] = pack(p[2 * e], p[2 * e + 1]);
      tc_store32(here, w);
      tc_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bar.p_ready));
      if (!(ok = tc_wait(&bar.dp_full, it & 1, deadline))) break;
      tc_fence_after();
      tc_load32(there, v[0]);
      tc_load32(there + 32, v[1]);
      tc_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bar.dp_free));
#pragma unroll
      for (int e = 0; e < 64; e += 4) {
        const float4 d = *reinterpret_cast<const float4 *>(delta + e);
        const float2 x = mul2(make_float2(p[e], p[e + 1]), add2(two(v, e), make_float2(d.x, d.y)));
        const float2 y = mul2(make_float2(p[e + 2], p[e + 3]), add2(two(v, e + 2), make_float2(d.z, d.w)));
        w[e / 2] = pack(x.x, x.y);
        w[e / 2 + 1] = pack(y.x, y.y);
      }
      tc_store32(here + 32, w);
      tc_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(smem_u32(&bar.ds_ready));
        mbar_arrive(smem_u32(&bar.line_empty[ls]));
      }
    }
    // warps 0-3 bring dv out, 4-7 dk, through shared memory that no product reads any more
    if (ok && total > 0) ok = tc_wait(&bar.done, (total - 1) & 1, deadline);
    if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
    tc_fence_after();
    const uint32_t from = tm + ((uint32_t)((warp & 3) * 32) << 16) + (half ? F::dk : F::dv);
    const float f = half ? z.scale : 1.0f;
    const View &out = half ? dk : dv;
    bf16 *dst = out.p + (long long)b * out.b + (long long)hk * out.h;
    uint8_t *tile = base + half * (ranks > 1 ? 2 : 1) * F::tile;
#pragma unroll
    for (int c = 0; c < 2 * NP; ++c) {
      uint32_t w[32] = {}, u[16];
      if (total > 0) {
        tc_load32(from + c * 32, w);
        tc_wait_ld();
      }
      if (ranks > 1) {
        keep_sums<NP>(tile, row, c * 32, w);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) u[e] = j < lk ? pack(__uint_as_float(w[2 * e]) * f, __uint_as_float(w[2 * e + 1]) * f) : 0u;
        stage_row<NP>(tile, row, c * 32, u);
      }
    }
    __syncwarp();
    if (ranks == 1) write_rows<NP>(tile, (warp & 3) * 32, j0, z.tk, z, dst, out.t);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) { tc_fence_after(); tc_free(tm, 512); }
  if (ranks > 1) {
    cluster_sync();
    if (warp < 8) {
      const int half = warp >> 2;
      const View &out = half ? dk : dv;
      join_sums<NP>(sk + half * 2 * F::tile, ranks, rank, threadIdx.x & 127, 128, j0, z.tk, lk, z, half ? z.scale : 1.0f,
                    out.p + (long long)b * out.b + (long long)hk * out.h, out.t);
    }
    cluster_sync();            // no CTA leaves while another reads its sums
  }
}

// dq of 128 queries of a head: dq += dS K over the key tiles it sees, S = Q K^T, dP = dO V^T.  A pass of its
// own: adding dq's parts up from the kernel above would need additions to memory in no fixed order.
// Tensor memory: S at 0, dP at 128, dq at 256, dS in turn at 384 and 448.
// The exponentials of one key tile are formed together with dS of the one before, so that the special
// function units work while the FMA units do.
constexpr int kDqThreads = 384;        // three warpgroups: 168 registers a thread at launch, 64,512 in all
template <int NP> struct Dq {
  static constexpr uint32_t tile = kT * 128 * NP;
  static constexpr int k_ring = NP == 1 ? 6 : 3, v_ring = NP == 1 ? 4 : 2;
  static constexpr uint32_t bars = (2 + k_ring + v_ring) * tile;
  static constexpr size_t smem = bars + 256;
  static constexpr uint32_t dq = 256, ds = 384;
};
template <int NP> struct DqBars {
  uint64_t q_full, k_full[Dq<NP>::k_ring], k_empty[Dq<NP>::k_ring], v_full[Dq<NP>::v_ring], v_empty[Dq<NP>::v_ring], s_full, s_free,
      dp_full, dp_free, ds_ready, dq_done[2];
  uint32_t tmem;
};

template <int NP>
__global__ void __launch_bounds__(kDqThreads, 1)
attn_backward_q(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo, const Sizes z,
                const float *__restrict__ lines, int padded, const View dq) {
  typedef Dq<NP> F;
  extern __shared__ __align__(1024) uint8_t base[];
  static_assert(sizeof(DqBars<NP>) <= 256, "barriers behind the tiles");
  DqBars<NP> &bar = *reinterpret_cast<DqBars<NP> *>(base + F::bars);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t sq = smem_u32(base), sdo = sq + F::tile, sk = sdo + F::tile, sv = sk + F::k_ring * F::tile;
  const int ranks = (int)cluster_size(), rank = (int)cluster_rank();
  const int column = blockIdx.x / ranks, h = column % z.heads, b = column / z.heads, hk = h / z.group;
  const int i0 = (z.causal ? (int)gridDim.y - 1 - (int)blockIdx.y : (int)blockIdx.y) * kT;

  if (threadIdx.x == 0) {
    if (sq & 1023u) atomicOr(z.status, CDG_ST_TIMEOUT);
    mbar_init(smem_u32(&bar.q_full), 1);
    for (int i = 0; i < F::k_ring; ++i) { mbar_init(smem_u32(&bar.k_full[i]), 1); mbar_init(smem_u32(&bar.k_empty[i]), 1); }
    for (int i = 0; i < F::v_ring; ++i) { mbar_init(smem_u32(&bar.v_full[i]), 1); mbar_init(smem_u32(&bar.v_empty[i]), 1); }
    mbar_init(smem_u32(&bar.s_full), 1); mbar_init(smem_u32(&bar.dp_full), 1);
    mbar_init(smem_u32(&bar.s_free), 8); mbar_init(smem_u32(&bar.dp_free), 8);
    mbar_init(smem_u32(&bar.ds_ready), 8);
    mbar_init(smem_u32(&bar.dq_done[0]), 1); mbar_init(smem_u32(&bar.dq_done[1]), 1);
    mbar_init_fence();
  }
  if (warp == 9) tc_alloc(&bar.tmem, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = bar.tmem;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const long long deadline = clock64() + kCdgWaitCycles;

  const int lq = used(z.q_lens, b, z.tq), lk = used(z.kv_lens, b, z.tk);
  const int seen = i0 >= lq ? 0 : z.causal ? min(lk, min(i0 + kT, lq) + lk - lq) : lk;
  const int all = seen > 0 && !(sq & 1023u) ? (seen + kT - 1) / kT : 0;
  const int total = (all - rank + ranks - 1) / ranks;        // this CTA's key tiles: rank, rank + ranks, ...

  if (warp >= 8) {
  tc_regs_down<56>();            // 128 x 56 + 256 x 224 = 64,512
  if (warp == 8) {
    if (tc_elect() && total > 0) {
      bool ok = true;
      int kn = 0, vn = 0;
      mbar_expect_tx(smem_u32(&bar.q_full), 2 * F::tile);
      load_tile<NP>(sq, &mq, i0, h, batch_of(z, kQ, b), smem_u32(&bar.q_full));
      load_tile<NP>(sdo, &mdo, i0, h, batch_of(z, kDo, b), smem_u32(&bar.q_full));
      for (int it = 0; it < total; ++it) {
        const int ks = it % F::k_ring, vs = it % F::v_ring, j0 = (rank + it * ranks) * kT;
        if (it >= F::k_ring && !(ok = mbar_wait(smem_u32(&bar.k_empty[ks]), (it / F::k_ring - 1) & 1, deadline))) break;
        mbar_expect_tx(smem_u32(&bar.k_full[ks]), F::tile);
        load_tile<NP>(sk + ks * F::tile, &mk, j0, hk, batch_of(z, kK, b), smem_u32(&bar.k_full[ks]));
        ++kn;
        if (it >= F::v_ring && !(ok = mbar_wait(smem_u32(&bar.v_empty[vs]), (it / F::v_ring - 1) & 1, deadline))) break;
        mbar_expect_tx(smem_u32(&bar.v_full[vs]), F::tile);
        load_tile<NP>(sv + vs * F::tile, &mv, j0, hk, batch_of(z, kV, b), smem_u32(&bar.v_full[vs]));
        ++vn;
      }
      if (!ok) {
        atomicOr(z.status, CDG_ST_TIMEOUT);
        mbar_wait(smem_u32(&bar.q_full), 0, clock64() + kCdgWaitCycles);
        for (int i = max(0, kn - F::k_ring); i < kn; ++i) mbar_wait(smem_u32(&bar.k_full[i % F::k_ring]), (i / F::k_ring) & 1, clock64() + kCdgWaitCycles);
        for (int i = max(0, vn - F::v_ring); i < vn; ++i) mbar_wait(smem_u32(&bar.v_full[i % F::v_ring]), (i / F::v_ring) & 1, clock64() + kCdgWaitCycles);
      }
    }
  } else if (warp == 9 || warp == 10) {
    auto arrived = [&](int it) {         // K of tile it, its rows past the sequence zeroed
      const int s = it % F::k_ring, left = lk - (rank + it * ranks) * kT;
      if (!tc_wait(&bar.k_full[s], (it / F::k_ring) & 1, deadline)) return false;
      if (z.kv_lens && left < kT) zero_rows<NP>(base + (sk - sq) + s * F::tile, left);
      return true;
    };
    auto scores = [&](int it) {          // S of tile it, when the one before is in registers
      if (!arrived(it) || (it > 0 && !tc_wait(&bar.s_free, (it - 1) & 1, deadline))) return false;
      tc_fence_after();
      if (tc_elect()) {
        mma_scores<NP>(tm, sq, sk + it % F::k_ring * F::tile);
        tc_commit(&bar.s_full);
      }
      __syncwarp();
      return true;
    };
    auto gradients = [&](int it) {       // dP likewise
      const int s = it % F::v_ring;
      if (!tc_wait(&bar.v_full[s], (it / F::v_ring) & 1, deadline) || (it > 0 && !tc_wait(&bar.dp_free, (it - 1) & 1, deadline))) return false;
      tc_fence_after();
      if (tc_elect()) {
        mma_scores<NP>(tm + kT, sdo, sv + s * F::tile);
        tc_commit(&bar.dp_full);
        tc_commit(&bar.v_empty[s]);
      }
      __syncwarp();
      return true;
    };
    bool ok = true;
    if (warp == 9) {
      ok = total == 0 || (tc_wait(&bar.q_full, 0, deadline) && scores(0));
      for (int it = 0; it < total && ok; ++it) ok = gradients(it) && (it + 1 == total || scores(it + 1));
    } else {
      for (int it = 0; it < total && ok; ++it) {
        const int ks = it % F::k_ring;
        if (!(ok = tc_wait(&bar.ds_ready, it & 1, deadline))) break;
        tc_fence_after();
        if (tc_elect()) {
          mma_rows<NP>(tm + F::dq, tm + F::ds + (it & 1) * 64, 32, sk + ks * F::tile, it > 0);
          tc_commit(&bar.dq_done[it & 1]);
          tc_commit(&bar.k_empty[ks]);
        }
        __syncwarp();
      }
    }
    if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
  }
  } else {
    tc_regs_up<224>();
    const int half = warp >> 2, row = (warp & 3) * 32 + lane, i = i0 + row;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, ts = tm + lanes + half * 64, tdp = ts + kT;
    const float a = z.negative ? -z.a : z.a;
    const int keys = i >= lq ? 0 : z.causal ? min(lk, i + lk - lq + 1) : lk;
    float l2 = -INFINITY, delta = 0.0f;          // both negated
    if (i < padded) {
      const float *line = lines + ((long long)b * z.heads + h) * 2 * padded + i;
      l2 = line[0];
      delta = line[padded];
    }
    const float2 aa = make_float2(a, a), ll = make_float2(l2, l2), dd = make_float2(delta, delta);
    bool ok = true;
    float p[64];
    if (total > 0 && (ok = tc_wait(&bar.s_full, 0, deadline))) {
      tc_fence_after();
      uint32_t v[2][32];
      tc_load32(ts, v[0]);
      tc_load32(ts + 32, v[1]);
      tc_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bar.s_free));
#pragma unroll
      for (int e = 0; e < 64; e += 2) {
        const float2 x = exp2_two<false>(fma2(two(v, e), aa, ll));
        p[e] = x.x;
        p[e + 1] = x.y;
      }
    }
    for (int it = 0; it < total && ok; ++it) {
      const bool next = it + 1 < total;
      if (!(ok = (!next || tc_wait(&bar.s_full, (it + 1) & 1, deadline)) && tc_wait(&bar.dp_full, it & 1, deadline))) break;
      tc_fence_after();
      uint32_t v[2][32] = {}, u[2][32], w[32];
      tc_load32(tdp, u[0]);
      tc_load32(tdp + 32, u[1]);
      if (next) {
        tc_load32(ts, v[0]);
        tc_load32(ts + 32, v[1]);
      }
      tc_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(smem_u32(&bar.dp_free));
        if (next) mbar_arrive(smem_u32(&bar.s_free));
      }
      const int left = keys - (rank + it * ranks) * kT - half * 64;
      if (__any_sync(0xffffffffu, left < 64)) {       // replaces P and dP: whatever lies there is not used
#pragma unroll
        for (int e = 0; e < 64; ++e)
          if (e >= left) { p[e] = 0.0f; u[e >> 5][e & 31] = 0u; }
      }
#pragma unroll
      for (int e = 0; e < 64; e += 2) {
        const float2 x = mul2(make_float2(p[e], p[e + 1]), add2(two(u, e), dd));
        w[e / 2] = pack(x.x, x.y);
        const float2 y = fma2(two(v, e), aa, ll), t = (e & 6) == 0 ? exp2_two<true>(y) : exp2_two<false>(y);
        p[e] = t.x;
        p[e + 1] = t.y;
      }
      if (it > 1) {              // the place of dS is free when its last product is over
        if (!(ok = tc_wait(&bar.dq_done[it & 1], (it / 2 - 1) & 1, deadline))) break;
        tc_fence_after();
      }
      tc_store32(tm + lanes + F::ds + (it & 1) * 64 + half * 32, w);
      tc_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bar.ds_ready));
    }
    if (ok && total > 0) ok = tc_wait(&bar.dq_done[(total - 1) & 1], ((total - 1) / 2) & 1, deadline);
    if (!ok && lane == 0) atomicOr(z.status, CDG_ST_TIMEOUT);
    tc_fence_after();
    // the two groups of warps bring out half of the head dimensions each, through the tiles of Q and dO
    const uint32_t from = tm + lanes + F::dq;
#pragma unroll
    for (int c = 0; c < NP; ++c) {
      const int col = (half * NP + c) * 32;
      uint32_t w[32] = {}, u[16];
      if (total > 0) {
        tc_load32(from + col, w);
        tc_wait_ld();
      }
      if (ranks > 1) {
        keep_sums<NP>(base, row, col, w);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) u[e] = keys > 0 ? pack(__uint_as_float(w[2 * e]) * z.scale, __uint_as_float(w[2 * e + 1]) * z.scale) : 0u;
        stage_row<NP>(base, row, col, u);
      }
    }
    asm volatile("bar.sync 1, 256;" ::: "memory");
    if (ranks == 1 && half == 0)
      write_rows<NP>(base, (warp & 3) * 32, i0, z.tq, z, dq.p + (long long)b * dq.b + (long long)h * dq.h, dq.t);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) { tc_fence_after(); tc_free(tm, 512); }
  if (ranks > 1) {
    cluster_sync();
    if (warp < 8)
      join_sums<NP>(sq, ranks, rank, threadIdx.x, 256, i0, z.tq, lq, z, z.scale, dq.p + (long long)b * dq.b + (long long)h * dq.h, dq.t);
    cluster_sync();
  }
}

// ---- host ---------------------------------------------------------------------------------------
constexpr long long kMaxStride = 1ll << 38;   // elements; a tensor map holds byte strides below 2^40

// strides of a tensor that is read: multiples of 16 bytes, tokens and heads apart from each other
bool in_ok(const long long s[3], int tokens, int heads, int dim) {
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] % 8 != 0 || s[i] > kMaxStride) return false;
  return (tokens <= 1 || s[1] >= dim) && (heads <= 1 || s[2] >= dim);
}
// ... and of one that is written: no two heads' values on top of each other
bool out_ok(const long long s[3], int batch, int tokens, int heads, int dim) {
  if (!in_ok(s, tokens, heads, dim)) return false;
  long long ext[3] = {batch, tokens, heads}, str[3] = {s[0], s[1], s[2]}, span = dim;
  for (int round = 0; round < 3; ++round) {
    int at = -1;                                    // the axis with the smallest stride that is left
    for (int i = 0; i < 3; ++i)
      if (ext[i] > 1 && (at < 0 || str[i] < str[at])) at = i;
    if (at < 0) return true;
    if (str[at] < span) return false;
    span += (ext[at] - 1) * str[at];
    ext[at] = 1;
  }
  return true;
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
  const int shared = (s->q_stride[0] > 0 ? 0 : kQ) | (s->k_stride[0] > 0 ? 0 : kK) | (s->v_stride[0] > 0 ? 0 : kV) |
                     (s->do_stride[0] > 0 ? 0 : kDo);
  return Sizes{s->batch, s->len_q, s->len_kv, s->heads, s->heads / s->kv_heads, s->head_dim, s->causal, s->scale,
               fmaxf(fabsf(s->scale) * kLog2e, 1e-30f), s->scale < 0.0f, shared, q_lens, kv_lens, status};
}
View view(const void *p, const long long s[3]) { return View{(bf16 *)const_cast<void *>(p), s[0], s[1], s[2]}; }

// [batch][head][token][dim] as the copies see it, boxes of 64 dimensions by 128 tokens
bool map_of(CUtensorMap *m, const void *p, const long long s[3], int batch, int tokens, int heads, int dim) {
  const long long dims[4] = {dim, tokens, heads, s[0] > 0 ? batch : 1};
  // an axis of length one (or shared by the batch, read at 0) still needs a stride the copy engine takes
  const long long strides[4] = {1, s[1] > 0 ? s[1] : 64, s[2] > 0 ? s[2] : 64, s[0] > 0 ? s[0] : 64};
  return tc_encode(m, true, p, 4, dims, strides, kT);
}
template <typename K>
bool raise_limit(CdgPerDevice &flags, K *kernel, size_t bytes) {
  int dev = 0;
  return cudaGetDevice(&dev) == cudaSuccess && cdg_raise_smem_limit(flags, dev, kernel, bytes) == cudaSuccess;
}

template <int NP>
int forward(const cdgrab_attention_shape *s, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const Sizes &z,
            const View &o, float *lse, cudaStream_t st) {
  static CdgPerDevice flags;
  if (!raise_limit(flags, attn_forward<NP>, Fwd<NP>::smem)) return CDGRAB_ERR_CUDA;
  return cdg_launch_rc(cdg_ops_launch(attn_forward<NP>, dim3(s->heads * s->batch, (s->len_q + 2 * kT - 1) / (2 * kT)), kFwdThreads,
                                      Fwd<NP>::smem, st, mq, mk, mv, z, o, lse));
}

// CTAs that share the loop of one tile of rows.  `longest` and `mean` are the turns of the loop for the
// longest tile and on average, `tiles` the number of tiles: a loop is dealt out while the longest one
// takes more than half of what every SM gets (so that the last CTAs to finish leave few SMs idle) and at
// least two turns are left to each CTA.
int split_of(double longest, double mean, double tiles, int sms) {
  int c = 1;
  while (c < 8 && longest / c > 0.5 * mean * tiles / sms && longest / (2 * c) >= 2.0) c *= 2;
  return c;
}
template <typename... KArgs, typename... Args>
int launch_cluster(void (*kernel)(KArgs...), dim3 grid, int cluster, int threads, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cdg_launch_rc(cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...));
}

template <int NP>
int backward(const cdgrab_attention_shape *s, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const CUtensorMap &mdo,
             const Sizes &z, const float *lines, int padded, const View &dq, const View &dk, const View &dv, int sms, cudaStream_t st) {
  static CdgPerDevice kf, qf;
  if (!raise_limit(kf, attn_backward_kv<NP>, Dkv<NP>::smem) || !raise_limit(qf, attn_backward_q<NP>, Dq<NP>::smem)) return CDGRAB_ERR_CUDA;
  int rc = CDGRAB_OK;
  const int qt = (s->len_q + kT - 1) / kT, kt = (s->len_kv + kT - 1) / kT;
  const double part = s->causal ? 0.5 : 1.0;
  if (kt > 0) {
    const int c = split_of((double)qt * z.group, part * qt * z.group, (double)kt * s->kv_heads * s->batch, sms);
    rc = launch_cluster(attn_backward_kv<NP>, dim3(s->kv_heads * s->batch * c, kt), c, kBwdThreads, Dkv<NP>::smem, st, mq, mk, mv, mdo, z,
                        lines, padded, dk, dv);
  }
  if (rc == CDGRAB_OK && qt > 0) {
    const int c = split_of(kt, part * kt, (double)qt * s->heads * s->batch, sms);
    rc = launch_cluster(attn_backward_q<NP>, dim3(s->heads * s->batch * c, qt), c, kDqThreads, Dq<NP>::smem, st, mq, mk, mv, mdo, z, lines,
                        padded, dq);
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
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const Sizes z = sizes_of(s, q_lens, kv_lens, dev->status);
  float *lines = (float *)workspace;
  const long long padded = ((long long)s->len_q + kT - 1) / kT * kT;
  if (s->len_q > 0) {
    const long long blocks = (s->batch * padded * s->heads * 8 + 255) / 256;
    if (blocks > 0x7fffffffll) return CDGRAB_ERR_INVALID;
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
