// Norms of queries and keys for each head and the rotation by the token's position, in one pass; and the backward pass,
// with the weights' gradients reduced per worker.
//
// Forward:   n = x rstd,  rstd = 1 / sqrt(sum x^2 / D + eps),  g = n w,  pairs of g turned by the angle t.
// Backward:  g' = the gradient turned by -t,  h = g' w,  dx = rstd (h - n (sum h n) / D),  dw = sum g' n.
// The angle of a far position is many turns: it is reduced in 64-bit integers, and only the fraction of a turn goes on in 32 bits.
#include <cmath>
#include <type_traits>

#include "ptx.cuh"
#include "rows.cuh"
#include "tensor_core.cuh"

namespace {

constexpr int kForward = 128, kBackward = 256;           // threads to a block
constexpr int kForwardResident = 7;        // blocks of the forward pass to an SM: 72 registers a thread (78 leave six blocks: 18.2 us for 15.6)
constexpr int kWarps = kBackward / 32;
constexpr int kResident = 2;               // blocks of the backward pass to an SM: 125 registers a thread
constexpr int kMaxDim = 256, kMaxPairs = kMaxDim / 2;
constexpr int kAhead = 4;                  // heads on their way

// Turns per position of each pair, base^(-2 i / rotary_dim) / (2 pi), less whole turns, in units of 2^-64, cut off: a position, which is
// whole, times that is the angle modulo a turn, to two units a position, in integer arithmetic that wraps.  (With a base below 1 the
// turns are many, and 64 bits hold less of their fraction.)
struct Frequencies { unsigned long long turns[kMaxPairs]; };

constexpr long double kPi = 3.14159265358979323846264338327950288L;

struct Side {                              // queries or keys
  const void *x, *dy;
  void *y;
  const float *w;
  long long xs[3], dys[3], ys[3];          // batch, token, head
  int heads;
};
struct Args {
  Side side[2];
  const void *pos;
  int pos_bits;
  long long pos_stride;
  const int *lens;
  CdgDivisor len, parts[2];                // tokens to a sequence; shares that a token's heads are dealt out in 
  int dim, rot, lanes, group;              // lanes: those that hold a head, V pairs each; group: the next power of two
  float eps;
};

// A group of lanes takes a token, or a share of its heads, head by head; the angles stay in registers meanwhile.
// A lane holds the values A = x[a .. a + V) and B = x[b .. b + V) of a head, one access each: V pairs, either (A_i, B_i), or
// (NEAR) neighbours, (A_2i, A_2i+1) and (B_2i, B_2i+1).  A and B lie in the halves of the rotated part, or of the rest.
template <int V>
__device__ __forceinline__ int2 places(const Args &a, int lane) {
  const int i = lane * V, half = a.rot / 2;
  if (i < half) return make_int2(i, half + i);
  return make_int2(a.rot + i - half, a.rot + (a.dim - a.rot) / 2 + i - half);
}

struct Shared {
  unsigned long long turns[kMaxPairs];     // of each lane's pairs, [V][lane]
  float weight[2][2][kMaxPairs];           // of queries and keys, A and B: [V / 4][lane][4]
  float sums[kWarps][kMaxDim], total[kMaxDim];
};

template <int V, bool NEAR>
__device__ __forceinline__ void load_shared(const Args &a, const Frequencies &f, Shared &s) {
  for (int i = threadIdx.x; i < a.lanes * V; i += blockDim.x) {
    const int lane = i / V, j = i % V, at = lane * V, half = a.rot / 2;
    // which pair of the head it is; one that stays turns by nothing
    const int pair = !NEAR ? at + j : j < V / 2 ? at / 2 + j : (half + at) / 2 + j - V / 2;
    s.turns[j * a.lanes + lane] = at < half ? f.turns[pair] : 0ull;
    const int2 p = places<V>(a, lane);
    const int to = (j / 4 * a.lanes + lane) * 4 + j % 4;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float *w = a.side[k].w;
      s.weight[k][0][to] = w ? w[p.x + j] : 1.0f;
      s.weight[k][1][to] = w ? w[p.y + j] : 1.0f;
    }
  }
}

// cos and sin of a lane's j-th angle at a position
template <int V>
__device__ __forceinline__ float2 angle(const Args &a, const Shared &sh, long long pos, int lane, int j) {
  const int part = (int)((unsigned long long)pos * sh.turns[j * a.lanes + lane] >> 32);      // of a turn, from -1/2
  float2 cs;
  sincospif((float)part * 0x1p-31f, &cs.y, &cs.x);
  return cs;
}

// What turns a lane's V pairs, in registers.  Halves: p c + q (-s), q c + p s; neighbours (x, y): (x, y) (c, c) + (y, x) (-s, s).
// Forward, the weight is in it: every factor times the weight of the value that it meets.
template <int V, bool NEAR>
struct Turn {
  float2 cp[V / 2], sp[V / 2], cq[V / 2], sq[V / 2];       // what p meets in p' and q', q in q' and p'; neighbours: p, swapped p, q, swapped q
  __device__ __forceinline__ void set(const Args &a, const Shared &sh, long long pos, int lane, const float *wa, const float *wb) {
#pragma unroll
    for (int j = 0; j < V; j += 2) {
      if (NEAR) {
        const float2 p = angle<V>(a, sh, pos, lane, j / 2), q = angle<V>(a, sh, pos, lane, V / 2 + j / 2);
        const float2 u = *reinterpret_cast<const float2 *>(wa + j / 4 * a.lanes * 4 + j % 4), v = *reinterpret_cast<const float2 *>(wb + j / 4 * a.lanes * 4 + j % 4);
        cp[j / 2] = make_float2(p.x * u.x, p.x * u.y);
        sp[j / 2] = make_float2(-p.y * u.y, p.y * u.x);
        cq[j / 2] = make_float2(q.x * v.x, q.x * v.y);
        sq[j / 2] = make_float2(-q.y * v.y, q.y * v.x);
      } else {
        const float2 k = angle<V>(a, sh, pos, lane, j), l = angle<V>(a, sh, pos, lane, j + 1);
        const float2 u = *reinterpret_cast<const float2 *>(wa + j / 4 * a.lanes * 4 + j % 4), v = *reinterpret_cast<const float2 *>(wb + j / 4 * a.lanes * 4 + j % 4);
        cp[j / 2] = make_float2(k.x * u.x, l.x * u.y);
        sp[j / 2] = make_float2(k.y * u.x, l.y * u.y);
        cq[j / 2] = make_float2(k.x * v.x, l.x * v.y);
        sq[j / 2] = make_float2(-k.y * v.x, -l.y * v.y);
      }
    }
  }
  __device__ __forceinline__ void apply(float2 (&p)[V / 2], float2 (&q)[V / 2]) const {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      if (NEAR) {
        p[j] = fma2(make_float2(p[j].y, p[j].x), sp[j], mul2(p[j], cp[j]));
        q[j] = fma2(make_float2(q[j].y, q[j].x), sq[j], mul2(q[j], cq[j]));
      } else {
        const float2 t = mul2(p[j], cp[j]);
        const float2 u = mul2(q[j], cq[j]);
        const float2 v = fma2(q[j], sq[j], t);
        q[j] = fma2(p[j], sp[j], u);
        p[j] = v;
      }
    }
  }
};
// The gradients turned back, without the weight: halves p c + q s, q c - p s.
template <int V, bool NEAR>
struct TurnBack {
  float2 c[NEAR ? V : V / 2], s[NEAR ? V : V / 2];
  __device__ __forceinline__ void set(const Args &a, const Shared &sh, long long pos, int lane) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float2 cs = angle<V>(a, sh, pos, lane, j);
      if (NEAR) {
        c[j] = make_float2(cs.x, cs.x);
        s[j] = make_float2(cs.y, -cs.y);
      } else if (j % 2) {
        c[j / 2].y = cs.x;
        s[j / 2].y = cs.y;
      } else {
        c[j / 2].x = cs.x;
        s[j / 2].x = cs.y;
      }
    }
  }
  __device__ __forceinline__ void apply(float2 (&p)[V / 2], float2 (&q)[V / 2]) const {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      if (NEAR) {
        p[j] = fma2(make_float2(p[j].y, p[j].x), s[j], mul2(p[j], c[j]));
        q[j] = fma2(make_float2(q[j].y, q[j].x), s[V / 2 + j], mul2(q[j], c[V / 2 + j]));
      } else {
        const float2 t = mul2(p[j], s[j]), u = mul2(q[j], c[j]);
        p[j] = fma2(q[j], s[j], mul2(p[j], c[j]));
        q[j] = make_float2(u.x - t.x, u.y - t.y);
      }
    }
  }
};

template <typename T, int V>
__device__ __forceinline__ void unpack(const CdgVec<T, V> &v, float2 (&p)[V / 2]) {
#pragma unroll
  for (int j = 0; j < V / 2; ++j) p[j] = make_float2(v.get(2 * j), v.get(2 * j + 1));
}
template <typename T, int V>
__device__ __forceinline__ void pack_store(const float2 (&p)[V / 2], T *to) {
  float f[V];
#pragma unroll
  for (int j = 0; j < V / 2; ++j) { f[2 * j] = p[j].x; f[2 * j + 1] = p[j].y; }
  CdgVec<T, V> v;
  v.set(f);
  v.store(to);
}
// A thread's own ring in shared memory: AHEAD stages of K accesses of V values, filled by asynchronous copies some heads ahead.
// A thread reads only what it copied, so the ring needs no barrier.  (What is on its way would fill the registers otherwise:
// with the next two or three heads in registers the forward pass took 22.6 and 21.5 us at 16 x 1024, 12 + 12 heads of 64.)
template <typename T, int V, int K, int AHEAD, int THREADS>
struct Ring {
  static constexpr int kBytes = V * sizeof(T);
  static constexpr size_t kSize = (size_t)AHEAD * K * THREADS * kBytes;
  uint32_t base;
  __device__ __forceinline__ explicit Ring(void *smem) : base(smem_u32(smem) + threadIdx.x * kBytes) {}
  __device__ __forceinline__ void copy(int stage, int k, const T *from) {
    const uint32_t to = base + (stage * K + k) * (THREADS * kBytes);
    if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
  }
  __device__ __forceinline__ static void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  // all but the last AHEAD - 1 commits have arrived
  __device__ __forceinline__ static void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 1) : "memory"); }
  __device__ __forceinline__ void read(int stage, int k, CdgVec<T, V> &v) const {
    const uint32_t at = base + (stage * K + k) * (THREADS * kBytes);
    if constexpr (kBytes == 16)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]) : "r"(at) : "memory");
    else
      asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.w[0]), "=r"(v.w[1]) : "r"(at) : "memory");
  }
};

// sum over a head's lanes
__device__ __forceinline__ float head_sum(float v, int group) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
    if (o < group) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// two at once
__device__ __forceinline__ float2 head_sums(float2 v, int group) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
    if (o < group) v = add2(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
  return v;
}

// A head on its way through the backward pass: a lane's values, their gradients turned back, times the weight.
template <int V>
struct Head {
  float2 p[V / 2], q[V / 2], g[V / 2], e[V / 2], ga[V / 2], gb[V / 2];
  // sum x^2 and sum h x: with x = n / rstd, both sums before rstd is known
  template <typename T, bool NEAR>
  __device__ __forceinline__ float2 sums(const CdgVec<T, V> &va, const CdgVec<T, V> &vb, const CdgVec<T, V> &da, const CdgVec<T, V> &db,
                                         const TurnBack<V, NEAR> &turn, const float *weight_a, const float *weight_b, int step, int group) {
    unpack(va, p); unpack(vb, q);
    unpack(da, g); unpack(db, e);
    turn.apply(g, e);
    float2 sum = make_float2(0.0f, 0.0f), along = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      sum = fma2(p[j], p[j], fma2(q[j], q[j], sum));
      ga[j] = mul2(g[j], p[j]);
      gb[j] = mul2(e[j], q[j]);
    }
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
      const float4 u = *reinterpret_cast<const float4 *>(weight_a + j * step), v = *reinterpret_cast<const float4 *>(weight_b + j * step);
      const float2 w[4] = {make_float2(u.x, u.y), make_float2(u.z, u.w), make_float2(v.x, v.y), make_float2(v.z, v.w)};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        along = fma2(ga[2 * j + i], w[i], fma2(gb[2 * j + i], w[2 + i], along));
        g[2 * j + i] = mul2(g[2 * j + i], w[i]);
        e[2 * j + i] = mul2(e[2 * j + i], w[2 + i]);
      }
    }
    return head_sums(make_float2(sum.x + sum.y, along.x + along.y), group);
  }
  // p, q: their gradients; the weights' sums with them
  __device__ __forceinline__ void finish(float square, float along, float inv, float2 (&wa)[V / 2], float2 (&wb)[V / 2]) {
    const float rstd = rsqrtf(square);
    const float off = -(along * inv * rstd * rstd) * rstd;
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      wa[j] = fma2(ga[j], make_float2(rstd, rstd), wa[j]);
      wb[j] = fma2(gb[j], make_float2(rstd, rstd), wb[j]);
      p[j] = fma2(p[j], make_float2(off, off), mul2(g[j], make_float2(rstd, rstd)));
      q[j] = fma2(q[j], make_float2(off, off), mul2(e[j], make_float2(rstd, rstd)));
    }
  }
};

// A head whose squares, or whose products with its gradient, may leave 32 bits although the results do not is brought to a size near
// one first: by a power of two, which changes no digit, taken from its largest value (or epsilon's root, so that epsilon stays in
// range with it).  n = x scale rstd,  1 / sqrt(sum x^2 / D + eps) = scale rstd.  Only the group's lanes take part.
// The loops over heads stop where a group of the warp has such a head, and the warp goes on in a loop of its own, so that the first one
// pays for the question alone: 2 to 3 % of the large backward pass (4 x 4096, 16 + 4 heads of 128: 50.2 us in a graph, 49.1 without), where a
// branch for each head took 4 to 6 %.
__device__ __forceinline__ unsigned group_lanes(int group) { return (0xffffffffu >> (32 - group)) << (threadIdx.x & 31 & ~(group - 1)); }
template <int V>
__device__ __forceinline__ float2 careful_norm(float2 (&p)[V / 2], float2 (&q)[V / 2], const Args &a) {
  const unsigned lanes = group_lanes(a.group);
  float most = sqrtf(a.eps);
#pragma unroll
  for (int j = 0; j < V / 2; ++j)
    most = fmaxf(most, fmaxf(fmaxf(fabsf(p[j].x), fabsf(p[j].y)), fmaxf(fabsf(q[j].x), fabsf(q[j].y))));
  for (int o = 1; o < a.group; o <<= 1) most = fmaxf(most, __shfl_xor_sync(lanes, most, o));
  const uint32_t exponent = min(max(__float_as_uint(most) >> 23, 1u), 253u);
  const float scale = __uint_as_float((254 - exponent) << 23);
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < V / 2; ++j) {
    p[j] = mul2(p[j], make_float2(scale, scale));
    q[j] = mul2(q[j], make_float2(scale, scale));
    sum += p[j].x * p[j].x + p[j].y * p[j].y + (q[j].x * q[j].x + q[j].y * q[j].y);
  }
  for (int o = 1; o < a.group; o <<= 1) sum += __shfl_xor_sync(lanes, sum, o);
  const float rstd = rsqrtf(sum / (float)a.dim + a.eps * scale * scale);
#pragma unroll
  for (int j = 0; j < V / 2; ++j) {
    p[j] = mul2(p[j], make_float2(rstd, rstd));
    q[j] = mul2(q[j], make_float2(rstd, rstd));
  }
  return make_float2(scale, rstd);
}
// The mean squares (epsilon included) between which the squares of a head lose nothing that counts.
constexpr float kForwardLow = 0x1p-60f, kForwardHigh = 0x1p120f;
// Backward, x takes the place of n until the norm is known, and its third power comes in.  With |x| up to sqrt(D) 2^12 and 1 / rstd
// from 2^-12 on, what products with the gradient lose below 2^-149 stays below 2^-122 times the weight in the results, and a sum up
// to kMostSum leaves room for the powers of rstd.
constexpr float kBackwardLow = 0x1p-24f, kBackwardHigh = 0x1p24f, kMostSum = 0x1p80f;

__device__ __forceinline__ long long position(const Args &a, uint32_t b, uint32_t t) {
  if (!a.pos) return t;
  const long long at = b * a.pos_stride + t;
  return a.pos_bits == 64 ? static_cast<const long long *>(a.pos)[at] : static_cast<const int *>(a.pos)[at];
}

// what is not in use: zeros, whatever epsilon and the weights are
template <typename T, int V>
__device__ __forceinline__ void store_zeros(T *y, long long step, int heads, int2 at) {
  const float2 none[V / 2] = {};
  for (int h = 0; h < heads; ++h, y += step) {
    pack_store<T, V>(none, y + at.x);
    pack_store<T, V>(none, y + at.y);
  }
}

// the first q_blocks blocks take queries, the others keys
template <typename T, int V, bool NEAR>
__global__ void __launch_bounds__(kForward, kForwardResident) rotary_forward_kernel(uint32_t tokens, uint32_t q_blocks, const __grid_constant__ Args a,
                                                                                    const __grid_constant__ Frequencies f) {
  extern __shared__ __align__(16) uint8_t dyn[];
  __shared__ __align__(16) Shared s;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int key = blockIdx.x >= q_blocks;
  const Side &z = a.side[key];
  const int group = a.group, lane = threadIdx.x & (group - 1);
  const bool mine = lane < a.lanes;
  const int2 at = places<V>(a, lane);
  const float inv = 1.0f / (float)a.dim;
  const uint32_t item = (blockIdx.x - (key ? q_blocks : 0)) * (kForward / group) + threadIdx.x / group;
  const bool some = item < tokens * a.parts[key].d;
  const uint32_t tok = some ? cdg_divide(item, a.parts[key]) : 0, share = item - tok * a.parts[key].d, b = cdg_divide(tok, a.len), t = tok - b * a.len.d;
  const int parts = a.parts[key].d, per = (z.heads + parts - 1) / parts, heads = some ? (z.heads - (int)share + parts - 1) / parts : 0;
  const bool used = some && (!a.lens || (int)t < a.lens[b]);
  const int count = used && mine ? heads : 0;
  const T *x = static_cast<const T *>(z.x) + b * z.xs[0] + t * z.xs[1] + share * z.xs[2];
  T *y = static_cast<T *>(z.y) + b * z.ys[0] + t * z.ys[1] + share * z.ys[2];
  const long long x_step = parts * z.xs[2], y_step = parts * z.ys[2];
  if (!used && mine) store_zeros<T, V>(y, y_step, heads, at);
  Ring<T, V, 2, kAhead, kForward> ring(dyn);
  auto request = [&](int h, int stage) {
    if (h < count) {
      ring.copy(stage, 0, x + at.x);
      ring.copy(stage, 1, x + at.y);
    }
    ring.commit();
    x += x_step;
  };
#pragma unroll
  for (int h = 0; h < kAhead - 1; ++h) request(h, h);
  load_shared<V, NEAR>(a, f, s);
  __syncthreads();
  Turn<V, NEAR> turn;
  turn.set(a, s, some ? position(a, b, t) : 0, mine ? lane : 0, s.weight[key][0] + (mine ? lane * 4 : 0), s.weight[key][1] + (mine ? lane * 4 : 0));
  int done = -1;                             // heads that are done where one needs care
  for (int h = 0, stage = 0; h < per; ++h, stage = stage + 1 == kAhead ? 0 : stage + 1) {      // (as often for every group)
    request(h + kAhead - 1, stage == 0 ? kAhead - 1 : stage - 1);
    ring.wait();
    CdgVec<T, V> va, vb;
    va.zero();
    vb.zero();
    if (h < count) {
      ring.read(stage, 0, va);
      ring.read(stage, 1, vb);
    }
    float2 p[V / 2], q[V / 2], sum = make_float2(0.0f, 0.0f);
    unpack(va, p);
    unpack(vb, q);
#pragma unroll
    for (int j = 0; j < V / 2; ++j) sum = fma2(p[j], p[j], fma2(q[j], q[j], sum));
    const float total = head_sum(sum.x + sum.y, group);
    const float square = total * inv + a.eps, rstd = rsqrtf(square);
    if (__any_sync(0xffffffffu, h < count && !(square >= kForwardLow && square <= kForwardHigh))) {
      done = h;
      break;
    }
    if (h >= count) continue;
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      p[j] = mul2(p[j], make_float2(rstd, rstd));
      q[j] = mul2(q[j], make_float2(rstd, rstd));
    }
    turn.apply(p, q);
    pack_store<T, V>(p, y + at.x);
    pack_store<T, V>(q, y + at.y);
    y += y_step;
  }
  if (__builtin_expect(done < 0, 1)) return;
  asm volatile("cp.async.wait_all;" ::: "memory");
  x = static_cast<const T *>(z.x) + b * z.xs[0] + t * z.xs[1] + share * z.xs[2];
  y = static_cast<T *>(z.y) + b * z.ys[0] + t * z.ys[1] + share * z.ys[2];
  for (int h = done; h < per; ++h) {
    const bool on = used && h < heads;
    CdgVec<T, V> va, vb;
    va.zero();
    vb.zero();
    if (on && mine) {
      va.load(x + h * x_step + at.x);
      vb.load(x + h * x_step + at.y);
    }
    float2 p[V / 2], q[V / 2], sum = make_float2(0.0f, 0.0f);
    unpack(va, p);
    unpack(vb, q);
#pragma unroll
    for (int j = 0; j < V / 2; ++j) sum = fma2(p[j], p[j], fma2(q[j], q[j], sum));
    const float square = head_sum(sum.x + sum.y, group) * inv + a.eps, rstd = rsqrtf(square);
    if (!on) continue;
    if (square >= kForwardLow && square <= kForwardHigh) {
#pragma unroll
      for (int j = 0; j < V / 2; ++j) {
        p[j] = mul2(p[j], make_float2(rstd, rstd));
        q[j] = mul2(q[j], make_float2(rstd, rstd));
      }
    } else {
      careful_norm<V>(p, q, a);
    }
    turn.apply(p, q);
    if (mine) {
      pack_store<T, V>(p, y + h * y_step + at.x);
      pack_store<T, V>(q, y + h * y_step + at.y);
    }
  }
}

// A block takes a chunk of one worker's (blockIdx.y) tokens, of its queries or of its keys, and keeps its sums of g' n in registers;
// at the end a cluster of blocks adds them up in order through distributed shared memory, and they go to the gradients, or, where
// a side has several clusters, to part[worker][cluster][dim], queries' first.
struct Grads {
  void *w[2];                              // of queries and keys, NULL: not wanted
  long long stride;                        // between workers
  int bf16;
  float *part;
};
template <typename T, int V, bool NEAR>
__global__ void __launch_bounds__(kBackward, kResident) rotary_backward_kernel(uint32_t tokens, int q_chunks, int k_chunks, const __grid_constant__ Args a,
                                                                      const __grid_constant__ Frequencies f, const __grid_constant__ Grads out) {
  __shared__ __align__(16) Shared s;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int key = blockIdx.x >= (unsigned)q_chunks, chunk = blockIdx.x - key * q_chunks, chunks = key ? k_chunks : q_chunks;
  const Side &z = a.side[key];
  const int group = a.group, groups = kBackward / group, lane = threadIdx.x & (group - 1);
  const bool mine = lane < a.lanes;
  const int2 at = places<V>(a, lane);
  const float inv = 1.0f / (float)a.dim;
  // each group an item; a side that is not there has none: its block only writes the zeros of its weight's gradient
  const uint32_t items = z.heads > 0 ? tokens * a.parts[key].d : 0, rounds = (items + groups - 1) / groups;
  const uint32_t r0 = (uint32_t)((unsigned long long)rounds * chunk / chunks), r1 = (uint32_t)((unsigned long long)rounds * (chunk + 1) / chunks);
  const int parts = a.parts[key].d, per = (z.heads + parts - 1) / parts;
  const long long x_step = parts * z.xs[2], dy_step = parts * z.dys[2], y_step = parts * z.ys[2];
  extern __shared__ __align__(16) uint8_t dyn[];
  Ring<T, V, 4, kAhead, kBackward> ring(dyn);
  float2 wa[V / 2] = {}, wb[V / 2] = {};
  load_shared<V, NEAR>(a, f, s);
  __syncthreads();
  const float *weight_a = s.weight[key][0] + (mine ? lane * 4 : 0), *weight_b = s.weight[key][1] + (mine ? lane * 4 : 0);
  uint32_t r = r0;
  int done = -1;                             // heads of the last item that are done where one needs care
  for (; r < r1; ++r) {
    const uint32_t item = r * groups + threadIdx.x / group;
    const bool some = item < items;
    const uint32_t local = some ? cdg_divide(item, a.parts[key]) : 0, share = item - local * a.parts[key].d;
    const uint32_t tok = blockIdx.y * tokens + local, b = cdg_divide(tok, a.len), t = tok - b * a.len.d;
    const int heads = some ? (z.heads - (int)share + parts - 1) / parts : 0;
    const bool used = some && (!a.lens || (int)t < a.lens[b]);
    const int count = used && mine ? heads : 0;
    const T *x = static_cast<const T *>(z.x) + b * z.xs[0] + t * z.xs[1] + share * z.xs[2];
    const T *dy = static_cast<const T *>(z.dy) + b * z.dys[0] + t * z.dys[1] + share * z.dys[2];
    T *y = static_cast<T *>(z.y) + b * z.ys[0] + t * z.ys[1] + share * z.ys[2];
    if (!used && mine) store_zeros<T, V>(y, y_step, heads, at);
    auto request = [&](int h, int stage) {
      if (h < count) {
        ring.copy(stage, 0, x + at.x);
        ring.copy(stage, 1, x + at.y);
        ring.copy(stage, 2, dy + at.x);
        ring.copy(stage, 3, dy + at.y);
      }
      ring.commit();
      x += x_step;
      dy += dy_step;
    };
#pragma unroll
    for (int h = 0; h < kAhead - 1; ++h) request(h, h);
    TurnBack<V, NEAR> turn;
    turn.set(a, s, some ? position(a, b, t) : 0, mine ? lane : 0);
    for (int h = 0, stage = 0; h < per; ++h, stage = stage + 1 == kAhead ? 0 : stage + 1) {
      request(h + kAhead - 1, stage == 0 ? kAhead - 1 : stage - 1);
      ring.wait();
      CdgVec<T, V> va, vb, da, db;
      va.zero(); vb.zero(); da.zero(); db.zero();
      if (h < count) {
        ring.read(stage, 0, va);
        ring.read(stage, 1, vb);
        ring.read(stage, 2, da);
        ring.read(stage, 3, db);
      }
      Head<V> head;
      const float2 both = head.sums(va, vb, da, db, turn, weight_a, weight_b, a.lanes * 4, group);
      const float square = both.x * inv + a.eps;
      const bool fits = square >= kBackwardLow && square <= kBackwardHigh && fabsf(both.y) <= kMostSum;
      if (__any_sync(0xffffffffu, h < count && !fits)) {
        done = h;
        break;
      }
      if (h >= count) continue;
      head.finish(square, both.y, inv, wa, wb);
      pack_store<T, V>(head.p, y + at.x);
      pack_store<T, V>(head.q, y + at.y);
      y += y_step;
    }
    if (done >= 0) break;
  }
  // From the first head on that needs care in any of a warp's groups, the warp goes on here.
  if (__builtin_expect(done >= 0, 0)) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    for (; r < r1; ++r, done = 0) {
      const uint32_t item = r * groups + threadIdx.x / group;
      const bool some = item < items;
      const uint32_t local = some ? cdg_divide(item, a.parts[key]) : 0, share = item - local * a.parts[key].d;
      const uint32_t tok = blockIdx.y * tokens + local, b = cdg_divide(tok, a.len), t = tok - b * a.len.d;
      const int heads = some ? (z.heads - (int)share + parts - 1) / parts : 0;
      const bool used = some && (!a.lens || (int)t < a.lens[b]);
      const T *x = static_cast<const T *>(z.x) + b * z.xs[0] + t * z.xs[1] + share * z.xs[2];
      const T *dy = static_cast<const T *>(z.dy) + b * z.dys[0] + t * z.dys[1] + share * z.dys[2];
      T *y = static_cast<T *>(z.y) + b * z.ys[0] + t * z.ys[1] + share * z.ys[2];
      if (!used && mine && done == 0) store_zeros<T, V>(y, y_step, heads, at);
      TurnBack<V, NEAR> turn;
      turn.set(a, s, some ? position(a, b, t) : 0, mine ? lane : 0);
      for (int h = done; h < per; ++h) {
        const bool on = used && h < heads;
        CdgVec<T, V> va, vb, da, db;
        va.zero(); vb.zero(); da.zero(); db.zero();
        if (on && mine) {
          va.load(x + h * x_step + at.x);
          vb.load(x + h * x_step + at.y);
          da.load(dy + h * dy_step + at.x);
          db.load(dy + h * dy_step + at.y);
        }
        Head<V> head;
        const float2 both = head.sums(va, vb, da, db, turn, weight_a, weight_b, a.lanes * 4, group);
        const float square = both.x * inv + a.eps;
        if (!on) continue;
        if (square >= kBackwardLow && square <= kBackwardHigh && fabsf(both.y) <= kMostSum) {
          head.finish(square, both.y, inv, wa, wb);
        } else {
          // in the formula's own order: the norm, then the products with n
          const float2 norm = careful_norm<V>(head.p, head.q, a);
          // (the gradient is read again: kept, it would take registers from the loop above)
          CdgVec<T, V> dc, dd;
          dc.zero(); dd.zero();
          if (mine) {
            dc.load(dy + h * dy_step + at.x);
            dd.load(dy + h * dy_step + at.y);
          }
          float2 g[V / 2], e[V / 2];
          unpack(dc, g); unpack(dd, e);
          turn.apply(g, e);
          float sum = 0.0f;
#pragma unroll
          for (int j = 0; j < V / 2; ++j) {
            wa[j] = fma2(g[j], head.p[j], wa[j]);
            wb[j] = fma2(e[j], head.q[j], wb[j]);
            sum += head.g[j].x * head.p[j].x + head.g[j].y * head.p[j].y + (head.e[j].x * head.q[j].x + head.e[j].y * head.q[j].y);
          }
          for (int o = 1; o < group; o <<= 1) sum += __shfl_xor_sync(group_lanes(group), sum, o);
          const float2 mean = make_float2(-sum * inv, -sum * inv), scale = make_float2(norm.x, norm.x), rstd = make_float2(norm.y, norm.y);
#pragma unroll
          for (int j = 0; j < V / 2; ++j) {
            head.p[j] = mul2(mul2(fma2(head.p[j], mean, head.g[j]), rstd), scale);
            head.q[j] = mul2(mul2(fma2(head.q[j], mean, head.e[j]), rstd), scale);
          }
        }
        if (mine) {
          pack_store<T, V>(head.p, y + h * y_step + at.x);
          pack_store<T, V>(head.q, y + h * y_step + at.y);
        }
      }
    }
  }
  if (!out.w[0] && !out.w[1]) return;
  // the groups of a warp, then the warps, then the blocks, in order
#pragma unroll
  for (int j = 0; j < V / 2; ++j) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      if (o >= group) {
        wa[j] = add2(wa[j], make_float2(__shfl_xor_sync(0xffffffffu, wa[j].x, o), __shfl_xor_sync(0xffffffffu, wa[j].y, o)));
        wb[j] = add2(wb[j], make_float2(__shfl_xor_sync(0xffffffffu, wb[j].x, o), __shfl_xor_sync(0xffffffffu, wb[j].y, o)));
      }
    if (mine && (threadIdx.x & 31) < group) {
      float *to = s.sums[threadIdx.x >> 5];
      to[at.x + 2 * j] = wa[j].x;
      to[at.x + 2 * j + 1] = wa[j].y;
      to[at.y + 2 * j] = wb[j].x;
      to[at.y + 2 * j + 1] = wb[j].y;
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < a.dim; c += kBackward) {
    float t = 0.0f;
    for (int o = 0; o < kWarps; ++o) t += s.sums[o][c];
    s.total[c] = t;
  }
  __syncthreads();
  const uint32_t ctas = tc_cluster_size(), rank = tc_cluster_rank();
  if (ctas > 1) tc_cluster_sync();
  const int clusters = chunks / (int)ctas;
  for (int c = (int)rank + threadIdx.x * (int)ctas; c < a.dim; c += kBackward * (int)ctas) {
    float t = 0.0f;
    for (uint32_t o = 0; o < ctas; ++o) {
      uint32_t there;
      float v;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(smem_u32(&s.total[c])), "r"(o));
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(there) : "memory");
      t += v;
    }
    if (clusters > 1) {
      out.part[((long long)blockIdx.y * (gridDim.x / ctas) + blockIdx.x / ctas) * a.dim + c] = t;
    } else if (out.w[key]) {
      const long long to = blockIdx.y * out.stride + c;
      if (out.bf16) static_cast<__nv_bfloat16 *>(out.w[key])[to] = __float2bfloat16_rn(t);
      else static_cast<float *>(out.w[key])[to] = t;
    }
  }
  __syncthreads();
  if (ctas > 1) tc_cluster_sync();                     // (no block leaves while another reads from it)
}

// the clusters' sums of one worker (blockIdx.y) added up in order, of queries (blockIdx.z = 0) or keys: 32 columns to a block, 32
// threads to a column.  A side with one has written its own.
constexpr int kJoinThreads = 1024, kJoinWarps = kJoinThreads / 32;
template <typename G>
__global__ void __launch_bounds__(kJoinThreads) rotary_join_kernel(int q_clusters, int k_clusters, int dim, const __grid_constant__ Grads out) {
  __shared__ float sm[kJoinWarps][33];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), k0 = threadIdx.x >> 5, key = blockIdx.z, clusters = key ? k_clusters : q_clusters;
  if (!out.w[key] || clusters < 2) return;
  const float *part = out.part + ((long long)blockIdx.y * (q_clusters + k_clusters) + (key ? q_clusters : 0)) * dim;
  float t = 0.0f;
  if (c < dim)
#pragma unroll 8
    for (int k = k0; k < clusters; k += kJoinWarps) t += part[(long long)k * dim + c];
  sm[k0][threadIdx.x & 31] = t;
  __syncthreads();
  if (k0 == 0 && c < dim) {
    for (int k = 1; k < kJoinWarps; ++k) t += sm[k][threadIdx.x];
    static_cast<G *>(out.w[key])[blockIdx.y * out.stride + c] = cdg_cast<G>(t);
  }
}

constexpr long long kMaxStride = 1ll << 40;

bool shape_ok(const cdgrab_rotary_shape *s) {
  return s && s->batch >= 0 && s->len >= 0 && s->heads >= 0 && s->kv_heads >= 0 && s->heads <= 65535 && s->kv_heads <= 65535 &&
         s->head_dim >= 8 && s->head_dim <= kMaxDim && s->head_dim % 8 == 0 && s->rotary_dim >= 0 && s->rotary_dim <= s->head_dim &&
         s->rotary_dim % 8 == 0 && (s->interleaved == 0 || s->interleaved == 1) && cdg_dtype_ok(s->dtype) && s->base > 0.0 &&
         std::isfinite(s->base) && s->eps >= 0.0f && std::isfinite(s->eps) && s->reserved == 0 && (long long)s->batch * s->len < (1ll << 31) &&
         (long long)(s->heads + s->kv_heads) * s->head_dim < (1ll << 31);
}

// pairs to a lane: 16 bytes on either side, 8 where bf16 heads or their rotated part do not divide so
int pairs_to_lane(const cdgrab_rotary_shape *s) {
  return s->dtype == CDGRAB_BF16 && s->rotary_dim % 16 == 0 && s->head_dim % 16 == 0 ? 8 : 4;
}
int lanes_of(const cdgrab_rotary_shape *s) { return s->head_dim / 2 / pairs_to_lane(s); }
int group_of(const cdgrab_rotary_shape *s) {
  int group = 1;
  while (group < lanes_of(s)) group *= 2;
  return group;
}
// Forward: shares that each token's heads are dealt out in, one by one, so that neighbouring groups read neighbouring heads: as many
// as fill five blocks to an SM, a share for every two heads at most; each share computes the token's angles again.  (16 x 1024, 12 + 12
// heads of 64: 15.6 us in one share, 16.8 in two; in blocks of 256 threads 19.7, of 64 threads 17.9: a block's tokens are its grain.)
constexpr int kSms = 148;
int parts_of(const cdgrab_rotary_shape *s, int heads) {
  const long long tokens = (long long)s->batch * s->len, fill = 5ll * kSms * (kForward / group_of(s));
  const long long most = (heads + 1) / 2, want = tokens > 0 ? fill / tokens : 1, parts = want < most ? want : most;
  if (parts <= 1) return 1;
  const long long per = (heads + parts - 1) / parts;
  return (int)((heads + per - 1) / per);
}
// Backward: how each worker's queries and keys are dealt out.  About kChunk values to a block, an item to each group of lanes at
// least, but no more blocks than four rounds of what is resident at once.  (2 x 300, 4 + 1 heads of 256 fp32: 6.8 us with 4096 values
// to a block, 8.7 with 8192, 12.5 with 16,384.)
// Where neither side of a worker has more than kOne values, each is one cluster, which needs no second launch: 19 us a call instead
// of 23, although the eight blocks take 13 us of them and more blocks 8 (3 x 357, 6 + 2 heads of 80 fp32).  Larger ones run as blocks
// of their own: in clusters they wait for room for all eight (4 x 4096, 16 + 4 heads of 128: 57 us instead of 49).
// A token's heads are dealt out in shares of four or more only where the blocks would otherwise lack tokens: each share computes the
// token's angles again and waits for its first head (the first case: 17 us in shares of two heads, 13 in one).
struct Blocks { int q, k, cluster, parts[2]; };
constexpr int kChunk = 4096, kCluster = 8, kOne = 1 << 18;
Blocks blocks_of(const cdgrab_rotary_shape *s, int m) {
  const long long tokens = (long long)s->batch / m * s->len, groups = kBackward / group_of(s);
  const long long most = 4ll * kResident * kSms / m < 1 ? 1 : 4ll * kResident * kSms / m, resident = 1ll * kResident * kSms / m < 1 ? 1 : 1ll * kResident * kSms / m;
  long long want[2];
  for (int i = 0; i < 2; ++i) want[i] = (tokens * (i ? s->kv_heads : s->heads) * s->head_dim + kChunk - 1) / kChunk;
  const bool one = (want[0] > want[1] ? want[0] : want[1]) * kChunk <= kOne;
  Blocks b = {1, 1, 1, {1, 1}};
  long long rounds[2] = {1, 1};
  for (int i = 0; i < 2; ++i) {
    const int heads = i ? s->kv_heads : s->heads;
    if (tokens == 0 || heads == 0) continue;
    const long long fill = one ? kCluster : want[i], blocks = fill < resident ? fill : resident, parts = blocks * groups / tokens, limit = (heads + 3) / 4;
    b.parts[i] = (int)(parts < 1 ? 1 : parts < limit ? parts : limit);
    const int per = (heads + b.parts[i] - 1) / b.parts[i];
    b.parts[i] = (heads + per - 1) / per;
    rounds[i] = (tokens * b.parts[i] + groups - 1) / groups;
  }
  if (one) {
    while (b.cluster < kCluster && (b.cluster < rounds[0] || b.cluster < rounds[1])) b.cluster *= 2;
    b.q = b.k = b.cluster;
  } else {
    for (int i = 0; i < 2; ++i) {
      const long long c = want[i] < most ? want[i] : most, n = c < rounds[i] ? c : rounds[i];
      (i ? b.k : b.q) = (int)(n < 1 ? 1 : n);
    }
  }
  return b;
}

void fill(const cdgrab_rotary_shape *s, Args &a, Frequencies &f) {
  for (int i = 0; i < 3; ++i) {
    a.side[0].xs[i] = s->q_stride[i]; a.side[1].xs[i] = s->k_stride[i];
    a.side[0].ys[i] = s->q_out_stride[i]; a.side[1].ys[i] = s->k_out_stride[i];
    a.side[0].dys[i] = s->dq_stride[i]; a.side[1].dys[i] = s->dk_stride[i];
  }
  a.side[0].heads = s->heads;
  a.side[1].heads = s->kv_heads;
  a.len = cdg_divisor((uint32_t)(s->len > 0 ? s->len : 1));
  a.lanes = lanes_of(s);
  a.group = group_of(s);
  a.dim = s->head_dim; a.rot = s->rotary_dim; a.eps = s->eps;
  // (a table of powers costs twice the rest of a small call: each thread keeps the last ones, replaced in turn)
  struct Kept { double base; int rot; Frequencies f; };
  static thread_local Kept kept[8] = {};
  static thread_local unsigned next = 0;
  const Kept *found = nullptr;
  for (const Kept &k : kept)
    if (k.base == s->base && k.rot == s->rotary_dim) found = &k;
  if (!found) {
    Kept &k = kept[next++ % 8];
    for (int i = 0; i < kMaxPairs; ++i) {
      long double whole, turns = 2 * i < s->rotary_dim ? std::pow((long double)s->base, -2.0L * i / s->rotary_dim) / (2.0L * kPi) : 0.0L;
      k.f.turns[i] = (unsigned long long)(std::modf(turns, &whole) * 0x1p64L);
    }
    k.base = s->base;
    k.rot = s->rotary_dim;
    found = &k;
  }
  f = found->f;
}

// f(T(), V, NEAR) for a shape's kernel
template <typename F>
int by_kind(const cdgrab_rotary_shape *s, F &&f) {
  auto near = [&](auto t, auto v) { return s->interleaved ? f(t, v, std::true_type()) : f(t, v, std::false_type()); };
  if (s->dtype == CDGRAB_F32) return near(0.0f, std::integral_constant<int, 4>());
  return pairs_to_lane(s) == 8 ? near(__nv_bfloat16(), std::integral_constant<int, 8>()) : near(__nv_bfloat16(), std::integral_constant<int, 4>());
}

// the checks that both directions share; backward: with the gradients
bool call_ok(const cdgrab_rotary_shape *s, const Args &a, bool backward) {
  const long long *in[] = {s->q_stride, s->k_stride, s->dq_stride, s->dk_stride}, *out[] = {s->q_out_stride, s->k_out_stride};
  for (int i = 0; i < (backward ? 4 : 2); ++i) {
    const int heads = i % 2 ? s->kv_heads : s->heads;
    if (heads > 0 && !cdg_heads_in_ok(in[i], s->len, heads, s->head_dim, kMaxStride)) return false;
  }
  for (int i = 0; i < 2; ++i) {
    const int heads = i ? s->kv_heads : s->heads;
    if (heads > 0 && !cdg_heads_out_ok(out[i], s->batch, s->len, heads, s->head_dim, kMaxStride)) return false;
  }
  for (int i = 0; i < 2; ++i) {
    const Side &z = a.side[i];
    if ((i ? s->kv_heads : s->heads) > 0 && (!z.x || !z.y || (backward && !z.dy))) return false;
    if (!cdg_aligned(z.x, 16) || !cdg_aligned(z.y, 16) || !cdg_aligned(z.dy, 16) || !cdg_aligned(z.w, 4)) return false;
  }
  if (!cdg_aligned(a.lens, 4)) return false;
  return !a.pos || ((a.pos_bits == 32 || a.pos_bits == 64) && a.pos_stride >= 0 && cdg_aligned(a.pos, a.pos_bits / 8));
}

}  // namespace

extern "C" int cdgrab_rotary_forward(const cdgrab_rotary_shape *s, const void *q, const void *k, const float *qw, const float *kw,
                                     const void *pos, int pos_bits, long long pos_stride, const int32_t *lens, void *qo, void *ko,
                                     void *stream) {
  if (!shape_ok(s)) return CDGRAB_ERR_INVALID;
  if (s->batch == 0 || s->len == 0 || s->heads + s->kv_heads == 0) return CDGRAB_OK;
  Args a = {};
  a.side[0].x = q; a.side[0].y = qo; a.side[0].w = qw;
  a.side[1].x = k; a.side[1].y = ko; a.side[1].w = kw;
  a.pos = pos; a.pos_bits = pos_bits; a.pos_stride = pos_stride; a.lens = lens;
  if (!call_ok(s, a, false)) return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  Frequencies f;
  fill(s, a, f);
  const long long tokens = (long long)s->batch * s->len;
  const int groups = kForward / a.group;
  unsigned blocks[2];
  for (int i = 0; i < 2; ++i) {
    const int heads = i ? s->kv_heads : s->heads;
    a.parts[i] = cdg_divisor(parts_of(s, heads));
    blocks[i] = heads ? (unsigned)((tokens * a.parts[i].d + groups - 1) / groups) : 0;
  }
  const dim3 grid(blocks[0] + blocks[1]);
  cudaStream_t st = (cudaStream_t)stream;
  return by_kind(s, [&](auto t, auto v, auto near) {
    using T = decltype(t);
    static CdgPerDevice flags;
    constexpr size_t smem = Ring<T, v(), 2, kAhead, kForward>::kSize;
    const cudaError_t e = cdg_raise_smem_limit(flags, dev->index, rotary_forward_kernel<T, v(), near()>, smem);
    return e != cudaSuccess ? cdg_launch_rc(e) : cdg_launch_rc(cdg_ops_launch(rotary_forward_kernel<T, v(), near()>, grid, kForward, smem, st,
                                                                              (uint32_t)tokens, blocks[0], a, f));
  });
}

extern "C" long long cdgrab_rotary_workspace_bytes(const cdgrab_rotary_shape *s, int m) {
  if (!shape_ok(s) || m < 1 || m > 65535 || s->batch % m) return -1;
  const Blocks b = blocks_of(s, m);
  return b.q == b.cluster && b.k == b.cluster ? 0 : 4ll * m * ((b.q + b.k) / b.cluster) * s->head_dim;
}

extern "C" int cdgrab_rotary_backward(const cdgrab_rotary_shape *s, int m, const void *dq, const void *dk, const void *q, const void *k,
                                      const float *qw, const float *kw, const void *pos, int pos_bits, long long pos_stride,
                                      const int32_t *lens, void *qo, void *ko, int grad_dtype, void *dqw, void *dkw,
                                      long long worker_stride, void *workspace, long long workspace_bytes, void *stream) {
  const long long need = cdgrab_rotary_workspace_bytes(s, m);
  if (need < 0 || !cdg_dtype_ok(grad_dtype)) return CDGRAB_ERR_INVALID;
  Args a = {};
  a.side[0].x = q; a.side[0].dy = dq; a.side[0].y = qo; a.side[0].w = qw;
  a.side[1].x = k; a.side[1].dy = dk; a.side[1].y = ko; a.side[1].w = kw;
  a.pos = pos; a.pos_bits = pos_bits; a.pos_stride = pos_stride; a.lens = lens;
  const long long tokens = (long long)s->batch / m * s->len;
  if (tokens > 0 && !call_ok(s, a, true)) return CDGRAB_ERR_INVALID;
  const int ge = grad_dtype == CDGRAB_F32 ? 4 : 2;
  if (((dqw || dkw) && m > 1 && worker_stride < s->head_dim) || !cdg_aligned(dqw, ge) || !cdg_aligned(dkw, ge)) return CDGRAB_ERR_INVALID;
  if (need > 0 && (!workspace || workspace_bytes < need || !cdg_aligned(workspace, 16))) return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  Frequencies f;
  fill(s, a, f);
  const Blocks n = blocks_of(s, m);
  for (int i = 0; i < 2; ++i) a.parts[i] = cdg_divisor(n.parts[i]);
  cudaStream_t st = (cudaStream_t)stream;
  const Grads out = {{dqw, dkw}, worker_stride, grad_dtype == CDGRAB_BF16, static_cast<float *>(workspace)};
  const int rc = by_kind(s, [&](auto t, auto v, auto near) {
    using T = decltype(t);
    static CdgPerDevice flags;
    constexpr size_t smem = Ring<T, v(), 4, kAhead, kBackward>::kSize;
    const cudaError_t e = cdg_raise_smem_limit(flags, dev->index, rotary_backward_kernel<T, v(), near()>, smem);
    return e != cudaSuccess ? cdg_launch_rc(e) : tc_launch_cluster(rotary_backward_kernel<T, v(), near()>, dim3(n.q + n.k, m), n.cluster, kBackward,
                                                                   smem, st, (uint32_t)tokens, n.q, n.k, a, f, out);
  });
  if (rc != CDGRAB_OK || (!dqw && !dkw) || (n.q == n.cluster && n.k == n.cluster)) return rc;
  const dim3 grid((s->head_dim + 31) / 32, m, 2);
  return cdg_launch_rc(out.bf16 ? cdg_ops_launch(rotary_join_kernel<__nv_bfloat16>, grid, kJoinThreads, 0, st, n.q / n.cluster, n.k / n.cluster, s->head_dim, out)
                                : cdg_ops_launch(rotary_join_kernel<float>, grid, kJoinThreads, 0, st, n.q / n.cluster, n.k / n.cluster, s->head_dim, out));
}
