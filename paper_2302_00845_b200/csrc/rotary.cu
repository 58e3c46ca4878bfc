// Norms of queries and keys for each head and the rotation by the token's position, in one pass; and the backward pass,
// with the weights' gradients reduced per worker.
//
// Forward:   n = x rstd,  rstd = 1 / sqrt(sum x^2 / D + eps),  g = n w,  pairs of g turned by the angle t.
// Backward:  g' = the gradient turned by -t,  h = g' w,  dx = rstd (h - n (sum h n) / D),  dw = sum g' n.
// The angle of a far position is many turns: position x (frequency / 2 pi) is taken in 64 bits and only its fraction
// goes on in 32.
#include <cmath>

#include "rows.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxDim = 256, kMaxPairs = kMaxDim / 2;
constexpr int kMaxTokens = 64;             // of a tile
constexpr int kMaxSlots = 2048;            // pairs of a tile

// turns per position of each pair: base^(-2 i / rotary_dim) / (2 pi), 0 for the pairs that stay
struct Frequencies { double turns[kMaxPairs]; };

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
  CdgDivisor len, lanes;                   // tokens to a sequence; lanes to a head, V pairs each
  CdgDivisor heads[3];                     // of queries, keys, both
  int dim, rot, interleaved, group, tile;  // group: lanes to a head, the next power of two; tile: tokens
  float eps;
};

// A lane holds the values A = x[a .. a + V) and B = x[b .. b + V) of a head, one access each: V pairs, either (A_i, B_i), or with
// neighbours in pairs (A_2i, A_2i+1) and (B_2i, B_2i+1).  Both halves of the rotated part, then both of the rest.
template <int V>
__device__ __forceinline__ int2 places(const Args &a, int lane) {
  const int i = lane * V, half = a.rot / 2;
  if (i < half) return make_int2(i, half + i);
  return make_int2(a.rot + i - half, a.rot + (a.dim - a.rot) / 2 + i - half);
}
// which pair of the head the lane's j-th is, -1 for one that stays
template <int V>
__device__ __forceinline__ int pair_of(const Args &a, int lane, int j) {
  const int i = lane * V, half = a.rot / 2;
  if (i >= half) return -1;
  if (!a.interleaved) return i + j;
  return j < V / 2 ? i / 2 + j : (half + i) / 2 + j - V / 2;
}

// What a tile of tokens shares, in shared memory.  Pieces of 16 bytes are kept lane after lane, so that a warp's reads meet no
// bank twice.
struct Tile {
  float2 turn[kMaxSlots];                  // cos and sin: [token][V / 2 pieces][lane][2 pairs]
  float weight[2][2][kMaxPairs];           // of queries and keys, A and B: [V / 4 pieces][lane][4]
  long long at[kMaxTokens][2];             // batch and token
  int live[kMaxTokens];
};

template <int V>
__device__ __forceinline__ void load_weights(const Args &a, Tile &s) {
  const int lanes = a.lanes.d;
  for (int i = threadIdx.x; i < 2 * a.dim / 2; i += kThreads) {
    const int k = i >= a.dim / 2, slot = i - k * (a.dim / 2), lane = slot / V, j = slot % V;
    const int2 p = places<V>(a, lane);
    const int to = (j / 4 * lanes + lane) * 4 + j % 4;
    const float *w = a.side[k].w;
    s.weight[k][0][to] = w ? w[p.x + j] : 1.0f;
    s.weight[k][1][to] = w ? w[p.y + j] : 1.0f;
  }
}

// angles, places and lengths of `tokens` tokens from token `first` on
template <int V>
__device__ __forceinline__ void load_tile(const Args &a, const Frequencies &f, Tile &s, long long first, int tokens) {
  const int lanes = a.lanes.d, slots = lanes * V;
  for (int i = threadIdx.x; i < tokens * slots; i += kThreads) {
    const uint32_t q = cdg_divide(i / V, a.lanes);               // token
    const int lane = i / V - q * lanes, j = i % V;
    const uint32_t tok = (uint32_t)(first + q), b = cdg_divide(tok, a.len);
    const uint32_t t = tok - b * a.len.d;
    if (i - q * slots == 0) {
      s.at[q][0] = b;
      s.at[q][1] = t;
      s.live[q] = !a.lens || (int)t < a.lens[b];
    }
    float2 cs = make_float2(1.0f, 0.0f);
    const int p = pair_of<V>(a, lane, j);
    if (p >= 0) {
      const long long at = b * a.pos_stride + t;
      const double pos = !a.pos ? (double)t : a.pos_bits == 64 ? (double)static_cast<const long long *>(a.pos)[at]
                                                               : (double)static_cast<const int *>(a.pos)[at];
      const double turns = pos * f.turns[p];
      sincospif(2.0f * (float)(turns - rint(turns)), &cs.y, &cs.x);
    }
    s.turn[q * slots + (j / 2 * lanes + lane) * 2 + j % 2] = cs;
  }
}

// the pairs of (p, q) turned, or turned back
template <int V, bool BACK>
__device__ __forceinline__ void turn_pairs(const Args &a, const float2 *turn, float (&p)[V], float (&q)[V]) {
  const float4 *c = reinterpret_cast<const float4 *>(turn);
  const int lanes = a.lanes.d;
  auto rotate = [](float cos, float sin, float &x, float &y) {
    const float u = BACK ? fmaf(x, cos, y * sin) : fmaf(x, cos, -(y * sin));
    y = BACK ? fmaf(y, cos, -(x * sin)) : fmaf(y, cos, x * sin);
    x = u;
  };
#pragma unroll
  for (int j = 0; j < V; j += 2) {
    const float4 cs = c[j / 2 * lanes];
    if (a.interleaved) {
      float *v = j < V / 2 ? p : q;
      const int i = j < V / 2 ? 2 * j : 2 * j - V;
      rotate(cs.x, cs.y, v[i], v[i + 1]);
      rotate(cs.z, cs.w, v[i + 2], v[i + 3]);
    } else {
      rotate(cs.x, cs.y, p[j], q[j]);
      rotate(cs.z, cs.w, p[j + 1], q[j + 1]);
    }
  }
}

// times the weight
template <int V>
__device__ __forceinline__ void weigh(const Args &a, const float *weight, float (&p)[V]) {
  const float4 *c = reinterpret_cast<const float4 *>(weight);
#pragma unroll
  for (int j = 0; j < V; j += 4) {
    const float4 w = c[j / 4 * a.lanes.d];
    p[j] *= w.x; p[j + 1] *= w.y; p[j + 2] *= w.z; p[j + 3] *= w.w;
  }
}

// sum over a head's lanes
__device__ __forceinline__ float head_sum(float v, int group) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
    if (o < group) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A block takes a tile of tokens, all heads of queries and keys: the tile's angles once, then a group of lanes to a head.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) rotary_forward_kernel(long long tokens, const __grid_constant__ Args a,
                                                                  const __grid_constant__ Frequencies f) {
  constexpr int U = 2;                     // heads to a group at a time
  __shared__ __align__(16) Tile s;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const long long first = (long long)blockIdx.x * a.tile;
  const int count = (int)min((long long)a.tile, tokens - first), items = count * (int)a.heads[2].d;
  const int group = a.group, lane = threadIdx.x & (group - 1), groups = kThreads / group;
  const bool mine = lane < (int)a.lanes.d;
  const int2 at = places<V>(a, lane);
  load_weights<V>(a, s);
  load_tile<V>(a, f, s, first, count);
  __syncthreads();
  for (int i0 = 0; i0 < items; i0 += U * groups) {
    CdgVec<T, V> va[U], vb[U];
    T *y[U];
    int tok[U], key[U];
    bool live[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * groups + threadIdx.x / group;
      va[u].zero();
      vb[u].zero();
      y[u] = nullptr;
      tok[u] = key[u] = 0;
      live[u] = false;
      if (i < items) {
        tok[u] = cdg_divide(i, a.heads[2]);
        int h = i - tok[u] * (int)a.heads[2].d;
        key[u] = h >= a.side[0].heads;
        if (key[u]) h -= a.side[0].heads;
        const Side &z = key[u] ? a.side[1] : a.side[0];
        live[u] = s.live[tok[u]];
        const long long b = s.at[tok[u]][0], t = s.at[tok[u]][1];
        y[u] = static_cast<T *>(z.y) + b * z.ys[0] + t * z.ys[1] + h * z.ys[2];
        if (live[u] && mine) {
          const T *x = static_cast<const T *>(z.x) + b * z.xs[0] + t * z.xs[1] + h * z.xs[2];
          va[u].load(x + at.x);
          vb[u].load(x + at.y);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float p[V], q[V], sum = 0.0f;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        p[j] = va[u].get(j);
        q[j] = vb[u].get(j);
        sum = fmaf(p[j], p[j], fmaf(q[j], q[j], sum));
      }
      const float rstd = 1.0f / sqrtf(head_sum(sum, group) / (float)a.dim + a.eps);
      if (!y[u] || !mine) continue;
      if (live[u]) {
#pragma unroll
        for (int j = 0; j < V; ++j) { p[j] *= rstd; q[j] *= rstd; }
        weigh<V>(a, s.weight[key[u]][0] + lane * 4, p);
        weigh<V>(a, s.weight[key[u]][1] + lane * 4, q);
        turn_pairs<V, false>(a, s.turn + tok[u] * (int)a.lanes.d * V + lane * 2, p, q);
        va[u].set(p);
        vb[u].set(q);
      }
      va[u].store(y[u] + at.x);
      vb[u].store(y[u] + at.y);
    }
  }
}

// A block takes a chunk of one worker's tokens (blockIdx.y), of its queries or of its keys, tile by tile, and keeps its sums of
// g' n in registers; at the end they go to part[worker][chunk][dim], queries' chunks first.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) rotary_backward_kernel(long long tokens, int q_chunks, int k_chunks, const __grid_constant__ Args a,
                                                                   const __grid_constant__ Frequencies f, float *part) {
  __shared__ __align__(16) Tile s;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int key = (int)blockIdx.x >= q_chunks, chunk = blockIdx.x - key * q_chunks, chunks = key ? k_chunks : q_chunks;
  const Side &z = a.side[key];
  // tiles are dealt out evenly
  const long long tiles = (tokens + a.tile - 1) / a.tile, t0 = tiles * chunk / chunks, t1 = tiles * (chunk + 1) / chunks;
  const long long base = (long long)blockIdx.y * tokens;
  const int group = a.group, lane = threadIdx.x & (group - 1), groups = kThreads / group;
  const bool mine = lane < (int)a.lanes.d;
  const int2 at = places<V>(a, lane);
  const float inv = 1.0f / (float)a.dim;
  float wa[V] = {}, wb[V] = {};
  load_weights<V>(a, s);
  for (long long tile = t0; tile < t1; ++tile) {
    const long long first = tile * a.tile;
    const int count = (int)min((long long)a.tile, tokens - first), items = count * z.heads;
    __syncthreads();
    load_tile<V>(a, f, s, base + first, count);
    __syncthreads();
    for (int i0 = 0; i0 < items; i0 += groups) {
      const int i = i0 + threadIdx.x / group;
      CdgVec<T, V> va, vb, da, db;
      va.zero(); vb.zero(); da.zero(); db.zero();
      T *y = nullptr;
      int tok = 0;
      bool live = false;
      if (i < items) {
        tok = cdg_divide(i, a.heads[key]);
        const int h = i - tok * z.heads;
        const long long b = s.at[tok][0], t = s.at[tok][1];
        y = static_cast<T *>(z.y) + b * z.ys[0] + t * z.ys[1] + h * z.ys[2];
        live = s.live[tok];
        if (live && mine) {
          const T *x = static_cast<const T *>(z.x) + b * z.xs[0] + t * z.xs[1] + h * z.xs[2];
          const T *dy = static_cast<const T *>(z.dy) + b * z.dys[0] + t * z.dys[1] + h * z.dys[2];
          va.load(x + at.x); vb.load(x + at.y);
          da.load(dy + at.x); db.load(dy + at.y);
        }
      }
      float p[V], q[V], g[V], h[V], sum = 0.0f;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        p[j] = va.get(j); q[j] = vb.get(j);
        g[j] = da.get(j); h[j] = db.get(j);
        sum = fmaf(p[j], p[j], fmaf(q[j], q[j], sum));
      }
      // (0 where there is nothing: with eps = 0 it would be infinite)
      sum = head_sum(sum, group);
      const float rstd = live ? 1.0f / sqrtf(sum * inv + a.eps) : 0.0f;
      if (mine) turn_pairs<V, true>(a, s.turn + tok * (int)a.lanes.d * V + lane * 2, g, h);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        p[j] *= rstd; q[j] *= rstd;
        wa[j] = fmaf(g[j], p[j], wa[j]);
        wb[j] = fmaf(h[j], q[j], wb[j]);
      }
      float hn = 0.0f;
      if (mine) {
        weigh<V>(a, s.weight[key][0] + lane * 4, g);
        weigh<V>(a, s.weight[key][1] + lane * 4, h);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) hn = fmaf(g[j], p[j], fmaf(h[j], q[j], hn));
      hn = head_sum(hn, group) * inv;
      if (!y || !mine) continue;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        p[j] = rstd * fmaf(-hn, p[j], g[j]);
        q[j] = rstd * fmaf(-hn, q[j], h[j]);
      }
      va.set(p); vb.set(q);
      va.store(y + at.x);
      vb.store(y + at.y);
    }
  }
  if (!part) return;
  // the groups of a warp, then the warps, in order; the tile's memory is free by then
  __syncthreads();
  float *sums = reinterpret_cast<float *>(s.turn);               // [warp][dim]
#pragma unroll
  for (int j = 0; j < V; ++j) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      if (o >= group) {
        wa[j] += __shfl_xor_sync(0xffffffffu, wa[j], o);
        wb[j] += __shfl_xor_sync(0xffffffffu, wb[j], o);
      }
    if (mine && (threadIdx.x & 31) < group) {
      sums[(threadIdx.x >> 5) * a.dim + at.x + j] = wa[j];
      sums[(threadIdx.x >> 5) * a.dim + at.y + j] = wb[j];
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < a.dim; c += kThreads) {
    float t = 0.0f;
    for (int o = 0; o < kWarps; ++o) t += sums[o * a.dim + c];
    part[((long long)blockIdx.y * gridDim.x + blockIdx.x) * a.dim + c] = t;
  }
}

// the chunks' sums of one worker (blockIdx.y) added up in order, of queries (blockIdx.z = 0) or keys: 32 columns to a block, eight
// threads to a column
template <typename G>
__global__ void __launch_bounds__(kThreads) rotary_join_kernel(int q_chunks, int k_chunks, int dim, const float *__restrict__ part, G *dqw, G *dkw,
                                                               long long ws) {
  __shared__ float sm[kWarps][33];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), k0 = threadIdx.x >> 5, key = blockIdx.z;
  G *out = key ? dkw : dqw;
  if (!out) return;
  const int chunks = key ? k_chunks : q_chunks;
  part += ((long long)blockIdx.y * (q_chunks + k_chunks) + (key ? q_chunks : 0)) * dim;
  float t = 0.0f;
  if (c < dim)
#pragma unroll 8
    for (int k = k0; k < chunks; k += kWarps) t += part[(long long)k * dim + c];
  sm[k0][threadIdx.x & 31] = t;
  __syncthreads();
  if (k0 == 0 && c < dim) {
    for (int k = 1; k < kWarps; ++k) t += sm[k][threadIdx.x];
    out[(long long)blockIdx.y * ws + c] = cdg_cast<G>(t);
  }
}

bool strides_ok(const long long (&s)[3], int len, int heads, int dim) {
  if (heads == 0) return true;
  for (long long v : s)
    if (v < 0 || v % 8 || v > (1ll << 40)) return false;
  return (len <= 1 || s[1] >= dim) && (heads <= 1 || s[2] >= dim);
}

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
// tokens to a tile: at most `items` heads to each group of lanes, as far as the angles' room goes
int tile_of(const cdgrab_rotary_shape *s, int heads, int items) {
  const int lanes = s->head_dim / 2 / pairs_to_lane(s), room = kMaxSlots / (s->head_dim / 2) < kMaxTokens ? kMaxSlots / (s->head_dim / 2) : kMaxTokens;
  int group = 1;
  while (group < lanes) group *= 2;
  const int want = items * (kThreads / group) / heads;
  return want < 1 ? 1 : want < room ? want : room;
}
constexpr int kSms = 148;
// Chunks of a worker's tokens, for queries and keys: in proportion to their heads about two rounds of the blocks that are resident
// at once (four to an SM), a tile to each at least.
void chunks_of(const cdgrab_rotary_shape *s, int m, int tile, int &q, int &k) {
  const long long tiles = ((long long)s->batch / m * s->len + tile - 1) / tile;
  const int all = s->heads + s->kv_heads;
  auto share = [&](int heads) {
    if (heads == 0 || tiles == 0) return 1ll;
    const long long c = (8ll * kSms * heads + (long long)all * m - 1) / ((long long)all * m);
    return c < tiles ? c : tiles;
  };
  q = (int)share(s->heads);
  k = (int)share(s->kv_heads);
}
int backward_tile(const cdgrab_rotary_shape *s) {
  const int most = s->heads > s->kv_heads ? s->heads : s->kv_heads;
  return tile_of(s, most > 0 ? most : 1, 2);
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
  const int lanes = s->head_dim / 2 / pairs_to_lane(s), counts[3] = {s->heads, s->kv_heads, s->heads + s->kv_heads};
  a.lanes = cdg_divisor(lanes);
  for (int i = 0; i < 3; ++i) a.heads[i] = cdg_divisor(counts[i] > 0 ? counts[i] : 1);
  for (a.group = 1; a.group < lanes;) a.group *= 2;
  a.dim = s->head_dim; a.rot = s->rotary_dim; a.interleaved = s->interleaved; a.eps = s->eps;
  // (a power for each pair costs more than the launch: each thread keeps its last table)
  static thread_local struct { double base; int rot; Frequencies f; } last = {};
  if (last.base != s->base || last.rot != s->rotary_dim) {
    for (int i = 0; i < kMaxPairs; ++i)
      last.f.turns[i] = 2 * i < s->rotary_dim ? std::pow(s->base, -2.0 * i / s->rotary_dim) / (2.0 * M_PI) : 0.0;
    last.base = s->base;
    last.rot = s->rotary_dim;
  }
  f = last.f;
}

// the checks that both directions share; backward: with the gradients
bool call_ok(const cdgrab_rotary_shape *s, const Args &a, bool backward) {
  if (!strides_ok(s->q_stride, s->len, s->heads, s->head_dim) || !strides_ok(s->k_stride, s->len, s->kv_heads, s->head_dim) ||
      !strides_ok(s->q_out_stride, s->len, s->heads, s->head_dim) || !strides_ok(s->k_out_stride, s->len, s->kv_heads, s->head_dim))
    return false;
  if (backward && (!strides_ok(s->dq_stride, s->len, s->heads, s->head_dim) || !strides_ok(s->dk_stride, s->len, s->kv_heads, s->head_dim)))
    return false;
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
  a.tile = tile_of(s, s->heads + s->kv_heads, 4);
  const long long tokens = (long long)s->batch * s->len;
  const dim3 grid((unsigned)((tokens + a.tile - 1) / a.tile));
  cudaStream_t st = (cudaStream_t)stream;
  auto go = [&](auto *kernel) { return cdg_launch_rc(cdg_ops_launch(kernel, grid, kThreads, 0, st, tokens, a, f)); };
  if (s->dtype == CDGRAB_F32) return go(rotary_forward_kernel<float, 4>);
  return pairs_to_lane(s) == 8 ? go(rotary_forward_kernel<__nv_bfloat16, 8>) : go(rotary_forward_kernel<__nv_bfloat16, 4>);
}

extern "C" long long cdgrab_rotary_workspace_bytes(const cdgrab_rotary_shape *s, int m) {
  if (!shape_ok(s) || m < 1 || m > 65535 || s->batch % m) return -1;
  int q, k;
  chunks_of(s, m, backward_tile(s), q, k);
  return 4ll * m * (q + k) * s->head_dim;
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
  if (!workspace || workspace_bytes < need || !cdg_aligned(workspace, 16)) return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  Frequencies f;
  fill(s, a, f);
  a.tile = backward_tile(s);
  int qc, kc;
  chunks_of(s, m, a.tile, qc, kc);
  cudaStream_t st = (cudaStream_t)stream;
  float *part = dqw || dkw ? static_cast<float *>(workspace) : nullptr;
  auto go = [&](auto *kernel) { return cdg_launch_rc(cdg_ops_launch(kernel, dim3(qc + kc, m), kThreads, 0, st, tokens, qc, kc, a, f, part)); };
  int rc = s->dtype == CDGRAB_F32 ? go(rotary_backward_kernel<float, 4>)
           : pairs_to_lane(s) == 8 ? go(rotary_backward_kernel<__nv_bfloat16, 8>) : go(rotary_backward_kernel<__nv_bfloat16, 4>);
  if (rc != CDGRAB_OK || !part) return rc;
  const dim3 grid((s->head_dim + 31) / 32, m, 2);
  return cdg_launch_rc(grad_dtype == CDGRAB_F32
                           ? cdg_ops_launch(rotary_join_kernel<float>, grid, kThreads, 0, st, qc, kc, s->head_dim, part, (float *)dqw, (float *)dkw, worker_stride)
                           : cdg_ops_launch(rotary_join_kernel<__nv_bfloat16>, grid, kThreads, 0, st, qc, kc, s->head_dim, part,
                                            (__nv_bfloat16 *)dqw, (__nv_bfloat16 *)dkw, worker_stride));
}
