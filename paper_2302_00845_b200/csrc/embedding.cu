// Embedding lookup and its gradient, reduced per worker into the gather buffer.
//
//   y[r] = scale table[t_r];   dtable[i][v] = scale sum of dy[r] over worker i's rows r with t_r = v.
//
// The lookup is bound by memory: a row read (from L2 where tokens repeat) and a row written.  The gradient writes every row of
// every worker's table, most of them zero, and reads dy once.  It runs in three launches:
//   1. each worker's tokens are sorted by value, stably, by a cluster of its own, while the other blocks clear the tables;
//   2. runs of equal tokens are summed in the order of their positions, a warp to 16 sorted positions and up to 256 columns;
//   3. runs that go on over more than two such windows, which step 2 leaves as a sum for each window, are joined: eight warps take
//      every eighth window each, and their sums are added in order.
// The order of a sum depends on the tokens alone, not on the order in which blocks run, and nothing is added to memory by atomics.
#include <cmath>

#include "rows.cuh"
#include "tensor_core.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

struct Tokens {
  const void *p;
  int bits;
  long long stride, length, padding;
  int vocab;
  // token j of row g of the tokens
  __device__ __forceinline__ long long at(long long g, long long j) const {
    return bits == 64 ? static_cast<const long long *>(p)[g * stride + j] : static_cast<const int *>(p)[g * stride + j];
  }
  __device__ __forceinline__ bool valid(long long t) const { return t >= 0 && t < vocab && t != padding; }
};

// ---- lookup -------------------------------------------------------------------------------------------
// A group of lanes takes a row, as many as it has accesses of VEC values and 32 at most; kAhead accesses of a lane are on their
// way together.  (65,536 rows of 768 bf16: 24.0 us, 5.3 TB/s, in 32 registers; two rows to a group 25.7; accesses numbered through
// all rows and dealt out one by one, each with a division and a token of its own, 27.5.)
template <typename T, typename R, int VEC>
__global__ void __launch_bounds__(kThreads) lookup_kernel(uint32_t rows, int per_row, int group, CdgDivisor length, Tokens tok, float scale,
                                                          const T *__restrict__ table, long long ts, R *__restrict__ y, long long ys,
                                                          int *status) {
  constexpr int kAhead = VEC * (int)sizeof(T) > 16 ? 2 : 4;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int lane = threadIdx.x & (group - 1);
  const uint32_t r = blockIdx.x * (kThreads / group) + threadIdx.x / group;
  if (r >= rows) return;
  const uint32_t g = cdg_divide(r, length);
  const long long t = tok.at(g, r - g * length.d);
  const bool valid = tok.valid(t);
  if (!valid && t != tok.padding && lane == 0) atomicOr(status, CDG_ST_INDEX);
  const T *from = table + (valid ? t * ts : 0) + lane * VEC;
  R *to = y + r * ys + lane * VEC;
  const int step = group * VEC;
  for (int c = lane; c < per_row; c += group * kAhead) {
    CdgVec<T, VEC> v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      v[u].zero();
      v[u].load_if(valid && c + u * group < per_row, from + u * step);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      float f[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[e] = v[u].get(e) * scale;
      CdgVec<R, VEC> o;
      o.set(f);
      if (c + u * group < per_row) o.store(to + u * step);
    }
    from += kAhead * step;
    to += kAhead * step;
  }
}

// Rows that are no whole number of 8-value accesses, into a contiguous y: a thread takes eight adjacent values of y, in one row or
// two (rows have eight at least), read LV at a time and stored at once.  (33 x 3773 rows of 37 bf16: 6.6 us, row by row 25.)
template <typename T, typename R, int LV>
__global__ void __launch_bounds__(kThreads) lookup_flat_kernel(uint32_t rows, CdgDivisor cols, CdgDivisor length, Tokens tok, float scale,
                                                               const T *__restrict__ table, long long ts, R *__restrict__ y, int *status) {
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const long long base = (long long)blockIdx.x * (kThreads * 8), first = base / cols.d;
  const uint32_t off = (uint32_t)(base - first * cols.d) + threadIdx.x * 8, q = cdg_divide(off, cols), c = off - q * cols.d;
  const long long r = first + q;
  if (r >= rows) return;
  // the row that the values start in, and the next
  const T *from[2];
  bool valid[2];
  const int here = min(8u, cols.d - c), n = here < 8 && r + 1 >= rows ? here : 8;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    valid[k] = false;
    if (k == 0 || here < n) {
      const uint32_t row = (uint32_t)r + k, g = cdg_divide(row, length);
      const long long t = tok.at(g, row - g * length.d);
      valid[k] = tok.valid(t);
      if (!valid[k] && t != tok.padding && (k == 1 || c == 0)) atomicOr(status, CDG_ST_INDEX);
      from[k] = table + (valid[k] ? t * ts : 0) + (k ? -here : (int)c);
    }
  }
  if (here == n) from[1] = from[0];
  CdgVec<T, LV> v[8 / LV];
#pragma unroll
  for (int i = 0; i < 8 / LV; ++i) {
    const bool second = i * LV >= here;
    v[i].zero();
    v[i].load_if(i * LV < n && (second ? valid[1] : valid[0]), (second ? from[1] : from[0]) + i * LV);
  }
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = v[e / LV].get(e % LV) * scale;
  R *to = y + base + threadIdx.x * 8;
  if (n == 8) {
    CdgVec<R, 8> o;
    o.set(f);
    o.store(to);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) to[e] = cdg_cast<R>(f[e]);
  }
}

// ---- gradient, step 1: sorted tokens, cleared tables -------------------------------------------------------
// A cluster sorts a worker's n tokens by a stable radix sort, digits of up to 8 bits, least first: the shortest form whose
// result does not depend on timing.  Each CTA of the cluster owns a contiguous share of the positions.  In a pass a warp ranks its
// items by matching digits among its lanes, the warps' counts are added up in order, the CTAs learn one another's counts through
// distributed shared memory, and the items move to their places.  A share of up to 4096 items is held in registers during a pass;
// of a longer one the digits are counted first, then it goes tile by tile.  Items are (token, row) pairs in two buffers that stay
// in L2.  Tokens without a gradient sort behind the vocabulary.
constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kBins = 256;
constexpr int kRounds = 8;             // items to a thread in a tile, at most
constexpr int kTile = kSortThreads * kRounds;
constexpr long long kShare = 1024;    // items to a CTA while more CTAs can be had

struct Sort {
  Tokens tok;
  CdgDivisor length;
  int groups, n, passes, bits;         // rows and tokens to a worker; digits and their bits
  uint2 *items, *other;                // [m][n] each; the result is in items
  int *status;
};
struct Clear {
  void *p;                             // NULL: nothing is cleared
  int elem;
  long long worker_stride, row_stride, cols, vocab, rows_per_block, blocks_per_worker, blocks;
};

__device__ __forceinline__ uint32_t cluster_read(const uint32_t *mine, uint32_t rank) {
  uint32_t there, v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(smem_u32(mine)), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(there) : "memory");
  return v;
}

// the item at position i of worker w in the first pass, and in later ones
__device__ __forceinline__ uint2 first_item(const Sort &s, long long w, uint32_t i) {
  const uint32_t g = cdg_divide(i, s.length);
  const long long t = s.tok.at(w * s.groups + g, i - g * s.length.d);
  const bool valid = s.tok.valid(t);
  if (!valid && t != s.tok.padding) atomicOr(s.status, CDG_ST_INDEX);
  return make_uint2(valid ? (uint32_t)t : (uint32_t)s.tok.vocab, i);
}

__device__ void sort_worker(const Sort &s, long long w, uint32_t rank, uint32_t ctas) {
  __shared__ uint32_t hist[kBins];                       // this CTA's digits in the pass
  __shared__ uint32_t place[kBins];                      // where the next item of a digit goes
  __shared__ uint32_t count[kSortWarps][kBins + 1];      // of a tile, by warp; then of the warps before
  __shared__ uint32_t part[kBins / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, bins = 1 << s.bits;
  const uint32_t share = (s.n + ctas - 1) / ctas, begin = min((uint32_t)s.n, rank * share), end = min((uint32_t)s.n, begin + share);
  const uint32_t mask = bins - 1;
  const bool single = share <= (uint32_t)kTile;
  for (int pass = 0; pass < s.passes; ++pass) {
    const uint2 *from = ((s.passes - pass) & 1 ? s.other : s.items) + w * s.n;
    uint2 *to = ((s.passes - pass) & 1 ? s.items : s.other) + w * s.n;
    const int shift = pass * s.bits;
    uint2 it[kRounds];
    uint32_t at[kRounds];
    int rounds = 0;
    uint32_t mine = 0;                                   // this thread's first item
    // items from i0 on, 32 to a warp and round
    auto load = [&](uint32_t t0) {
      const uint32_t left = end - t0;
      rounds = left >= (uint32_t)kTile ? kRounds : (int)((left + kSortThreads - 1) / kSortThreads);
      mine = t0 + warp * rounds * 32 + lane;
#pragma unroll
      for (int r = 0; r < kRounds; ++r) {
        const uint32_t i = mine + r * 32;
        if (r < rounds && i < end) it[r] = pass == 0 ? first_item(s, w, i) : __ldcg(from + i);
      }
    };
    // each item's rank in its warp, counts of the warps before in count, the tile's digits in total (of thread d for digit d)
    auto rank_tile = [&]() {
      for (int d = lane; d < bins; d += 32) count[warp][d] = 0;
      __syncwarp();
#pragma unroll
      for (int r = 0; r < kRounds; ++r) {
        if (r >= rounds) break;
        const uint32_t d = mine + r * 32 < end ? it[r].x >> shift & mask : kBins;
        const uint32_t same = __match_any_sync(0xffffffffu, d);
        at[r] = 0;
        if (d < kBins) at[r] = count[warp][d] + __popc(same & ((1u << lane) - 1));
        __syncwarp();
        if (d < kBins && lane == __ffs(same) - 1) count[warp][d] += __popc(same);
        __syncwarp();
      }
      __syncthreads();
      uint32_t total = 0;
      if (tid < bins) {
        uint32_t c[kSortWarps];
#pragma unroll
        for (int k = 0; k < kSortWarps; ++k) c[k] = count[k][tid];
#pragma unroll
        for (int k = 0; k < kSortWarps; ++k) {
          count[k][tid] = total;
          total += c[k];
        }
      }
      return total;
    };
    auto scatter = [&]() {
#pragma unroll
      for (int r = 0; r < kRounds; ++r)
        if (r < rounds && mine + r * 32 < end) {
          const uint32_t d = it[r].x >> shift & mask;
          to[place[d] + count[warp][d] + at[r]] = it[r];
        }
    };
    uint32_t digits = 0;
    if (single) {
      load(begin);
      digits = rank_tile();
      if (tid < bins) hist[tid] = digits;
    } else {
      for (int d = tid; d < bins; d += kSortThreads) hist[d] = 0;
      __syncthreads();
      for (uint32_t t0 = begin; t0 < end; t0 += kTile) {
        load(t0);
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
          if (r >= rounds) break;
          const uint32_t d = mine + r * 32 < end ? it[r].x >> shift & mask : kBins;
          const uint32_t same = __match_any_sync(0xffffffffu, d);
          if (d < kBins && lane == __ffs(same) - 1) atomicAdd(&hist[d], __popc(same));
        }
      }
    }
    __syncthreads();
    if (ctas > 1) tc_cluster_sync();
    // a digit's first place: all items of lower digits, and this digit's of the CTAs before
    uint32_t total = 0, before = 0;
    if (tid < bins) {
      if (ctas > 1) {
        for (uint32_t c = 0; c < ctas; ++c) {
          const uint32_t h = cluster_read(&hist[tid], c);
          before += c < rank ? h : 0;
          total += h;
        }
      } else {
        total = hist[tid];
      }
    }
    uint32_t sum = total;
    if (tid < kBins) {
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += v;
      }
      if (lane == 31) part[warp] = sum;
    }
    __syncthreads();
    if (tid < bins) {
      uint32_t lower = sum - total + before;
      for (int k = 0; k < warp; ++k) lower += part[k];
      place[tid] = lower;
    }
    __syncthreads();
    if (single) {
      scatter();
    } else {
      for (uint32_t t0 = begin; t0 < end; t0 += kTile) {
        load(t0);
        digits = rank_tile();
        __syncthreads();
        scatter();
        __syncthreads();
        if (tid < bins) place[tid] += digits;
      }
    }
    __syncthreads();
    if (ctas > 1) tc_cluster_sync();
  }
}

// `bytes` zeros from p on, by the whole block
__device__ __forceinline__ void clear_span(uint8_t *p, long long bytes, int elem) {
  const int lead = (int)((32 - ((uintptr_t)p & 31)) & 31);
  if (bytes <= lead + 32) {
    for (long long i = (long long)threadIdx.x * elem; i < bytes; i += (long long)blockDim.x * elem) {
      if (elem == 4) *reinterpret_cast<uint32_t *>(p + i) = 0;
      else *reinterpret_cast<uint16_t *>(p + i) = 0;
    }
    return;
  }
  const long long body = (bytes - lead) & ~31ll, tail = bytes - lead - body;
  for (long long i = (long long)threadIdx.x * 32; i < body; i += (long long)blockDim.x * 32)
    asm volatile("st.global.v8.b32 [%0], {%1, %1, %1, %1, %1, %1, %1, %1};" ::"l"(p + lead + i), "r"(0) : "memory");
  const int i = threadIdx.x * 2;               // (both ends are shorter than 32 bytes and of whole elements)
  if (i < lead) *reinterpret_cast<uint16_t *>(p + i) = 0;
  if (i < tail) *reinterpret_cast<uint16_t *>(p + lead + body + i) = 0;
}

// (two blocks to an SM, 64 registers: with one, 16 tables of 50,257 x 768 bf16 are cleared 6 % slower)
__global__ void __launch_bounds__(kSortThreads, 2) sort_and_clear_kernel(const __grid_constant__ Sort s, const __grid_constant__ Clear z,
                                                                      unsigned sorting) {
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  if (blockIdx.x < sorting) {
    const uint32_t ctas = tc_cluster_size();
    sort_worker(s, blockIdx.x / ctas, tc_cluster_rank(), ctas);
    return;
  }
  for (long long b = blockIdx.x - sorting; b < z.blocks; b += gridDim.x - sorting) {
    const long long w = b / z.blocks_per_worker, v0 = (b - w * z.blocks_per_worker) * z.rows_per_block;
    const long long rows = min(z.rows_per_block, z.vocab - v0);
    uint8_t *p = static_cast<uint8_t *>(z.p) + (w * z.worker_stride + v0 * z.row_stride) * z.elem;
    if (z.row_stride == z.cols) {
      clear_span(p, rows * z.cols * z.elem, z.elem);
    } else {
      for (long long v = 0; v < rows; ++v) clear_span(p + v * z.row_stride * z.elem, z.cols * z.elem, z.elem);
    }
  }
}

// ---- gradient, steps 2 and 3: sums over runs of equal tokens -----------------------------------------------
// A window is kWindow sorted positions.  A run that starts in window w and ends in it or in the next one belongs to w, which sums all
// of it.  A longer one is summed window by window: its part in the window it starts in goes to part[w][0], its parts in the windows
// it goes on in to part[.][1].  Keys kWindow + 1 positions back and 2 kWindow ahead tell which case it is, without a search.
struct Sums {
  const uint2 *items;
  int n, windows, vocab, cols;
  float *part;                         // [m][windows][2][cols]
  const void *dy;
  long long dy_stride;
  void *dtable;
  long long worker_stride, row_stride;
  float scale;
  int accumulate;
};

constexpr uint32_t kNoKey = 0xffffffffu;
constexpr int kWindow = 16;            // half a warp: its lanes hold a window and the next one
constexpr int kSumThreads = 128;       // (a block stays until its longest window is done: with 256 the case below takes 53 us)

// A warp to a window and 32 VEC NV columns; kAhead rows are on their way together.  What bounds it is instructions, not memory: a
// warp goes through a few dozen rows in its life, so each case that is spelled out for each row in flight costs its fetching, and each
// predicate on a load its issue slots (2 x 7892 tokens of 1377 bf16 columns: 124 us with all cases for eight rows, predicated, 47 in a
// graph with sort and join so).
template <typename T, typename G, int VEC, int NV>
__global__ void __launch_bounds__(kSumThreads) run_sums_kernel(const __grid_constant__ Sums a, long long all) {
  constexpr int kAhead = 4, kSlab = 32 * VEC * NV;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int lane = threadIdx.x & 31;
  const long long at = (long long)blockIdx.x * (kSumThreads / 32) + (threadIdx.x >> 5);      // worker and window
  if (at >= all) return;
  const long long w = at / a.windows;
  const int win = (int)(at - w * a.windows);
  const long long p0 = (long long)win * kWindow;
  const uint2 *items = a.items + w * a.n;
  auto key = [&](long long p) { return p >= 0 && p < a.n ? items[p].x : kNoKey; };
  const uint2 e = p0 + lane < a.n ? items[p0 + lane] : make_uint2(kNoKey, 0u);
  const uint32_t back1 = key(p0 - 1), back2 = key(p0 - kWindow - 1), ahead = key(p0 + 2 * kWindow);
  const uint32_t first = __shfl_sync(0xffffffffu, e.x, 0), last = __shfl_sync(0xffffffffu, e.x, kWindow - 1);
  const uint32_t next = __shfl_sync(0xffffffffu, e.x, kWindow);
  constexpr uint32_t here = (1u << kWindow) - 1;
  // tokens without a gradient are past the others, and what is past the end behind them
  const int live = __popc(__ballot_sync(0xffffffffu, e.x < (uint32_t)a.vocab) & here);
  if (live == 0) return;
  const bool goes_on = first == back1;                                  // the first run began before
  const bool head_long = goes_on && (first == back2 || first == next);
  const int head = __popc(__ballot_sync(0xffffffffu, e.x == first) & here);      // its positions here
  const bool whole = head == kWindow && goes_on;                        // nothing begins here
  const uint32_t lasts = __ballot_sync(0xffffffffu, e.x == last);
  const bool tail_long = !whole && live == kWindow && last == ahead;
  const int begin = goes_on && !head_long ? head : 0;
  const int end = live + (!whole && live == kWindow && !tail_long ? __popc(lasts >> kWindow) : 0);
  if (begin >= end) return;
  // positions at which a run ends
  const uint32_t after = __shfl_down_sync(0xffffffffu, e.x, 1);
  const uint32_t ends = __ballot_sync(0xffffffffu, e.x != after);
  const int split = head_long ? head : begin;                           // a part of a longer run comes first, by itself
  for (int c0 = blockIdx.y * kSlab; c0 < a.cols; c0 += gridDim.y * kSlab) {
    const int c = c0 + lane * VEC;
    // (lanes past the last column read it again and keep nothing)
    const T *dy = static_cast<const T *>(a.dy) + w * a.n * a.dy_stride;
    int off[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) off[i] = min(c + i * 32 * VEC, a.cols - VEC);
    G *table = static_cast<G *>(a.dtable) + w * a.worker_stride + c;
    float *part = a.part + (w * a.windows + win) * 2 * (long long)a.cols + c;
    for (int half = head_long ? 0 : 1; half < 2; ++half) {
      const int from = half ? split : begin, to = half ? end : split;
      const bool piece = half ? tail_long : true;                       // the last run's sum is part of a longer one's
      float acc[NV][VEC] = {};
      CdgVec<T, VEC> v[kAhead][NV];
      auto load = [&](int q, CdgVec<T, VEC> (&row)[NV]) {
        const T *p = dy + __shfl_sync(0xffffffffu, e.y, min(q, to - 1)) * a.dy_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) row[i].load(p + off[i]);
      };
#pragma unroll
      for (int u = 0; u < kAhead; ++u) load(from + u, v[u]);
#pragma unroll 1
      for (int p = from; p < to; p += kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int q = p + u;
          if (q >= to) break;
#pragma unroll
          for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int f = 0; f < VEC; ++f) acc[i][f] += v[u][i].get(f);
          load(q + kAhead, v[u]);
          if (q + 1 < to ? ends >> q & 1 : !piece) {
            G *out = table + __shfl_sync(0xffffffffu, e.x, q) * a.row_stride;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
              CdgVec<G, VEC> o;
              float g[VEC];
              o.zero();
              o.load_if(a.accumulate && c + i * 32 * VEC < a.cols, out + i * 32 * VEC);
#pragma unroll
              for (int f = 0; f < VEC; ++f) {
                g[f] = fmaf(acc[i][f], a.scale, o.get(f));
                acc[i][f] = 0.0f;
              }
              o.set(g);
              o.store_if(c + i * 32 * VEC < a.cols, out + i * 32 * VEC);
            }
          }
        }
      }
      if (piece) {
        float *sum = half ? part : part + a.cols;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int f = 0; f < VEC; ++f)
            if (c + i * 32 * VEC < a.cols) sum[i * 32 * VEC + f] = acc[i][f];
      }
    }
  }
}

// A block to kJoin windows and 256 columns: the parts of each long run that starts there, warp q taking every eighth.
constexpr int kJoin = 8, kJoinCols = 256;
template <typename G>
__global__ void __launch_bounds__(kThreads) join_runs_kernel(const __grid_constant__ Sums a, long long all) {
  __shared__ float sm[kWarps][kJoinCols];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long at0 = (long long)blockIdx.x * kJoin;
  // which of the windows a long run starts in
  bool starts = false;
  if (lane < kJoin && at0 + lane < all) {
    const long long w = (at0 + lane) / a.windows, p0 = (at0 + lane - w * a.windows) * kWindow;
    const uint2 *items = a.items + w * a.n;
    if (p0 + 2 * kWindow < a.n) {
      const uint32_t k = items[p0 + kWindow - 1].x, ahead = items[p0 + 2 * kWindow].x, back = p0 > 0 ? items[p0 - 1].x : kNoKey;
      starts = k < (uint32_t)a.vocab && k == ahead && k != back;
    }
  }
  for (uint32_t todo = __ballot_sync(0xffffffffu, starts); todo; todo &= todo - 1) {
    const long long at = at0 + __ffs(todo) - 1, w = at / a.windows;
    const int win = (int)(at - w * a.windows);
    const uint2 *items = a.items + w * a.n;
    const uint32_t k = items[(long long)win * kWindow + kWindow - 1].x;
    // how many windows it reaches into: keys are sorted, so the last is bracketed by powers of two, then by 32 steps at a time
    auto holds = [&](long long v) { return win + v < a.windows && items[(win + v) * kWindow].x == k; };
    const int power = __popc(__ballot_sync(0xffffffffu, holds(1ll << lane)));        // 2^(power - 1) windows on still, 2^power not
    long long in = power ? 1ll << (power - 1) : 0, step = in;
    while (step > 1) {                       // in holds, in + step does not
      step = (step + 31) / 32;
      in += step * (__popc(__ballot_sync(0xffffffffu, holds(in + step * (lane + 1)))));
    }
    const int pieces = (int)in + 1;
    const float *part = a.part + (w * a.windows + win) * 2 * (long long)a.cols;
    for (int c0 = blockIdx.y * kJoinCols; c0 < a.cols; c0 += gridDim.y * kJoinCols) {
      float s[kJoinCols / 32] = {};
#pragma unroll 4
      for (int v = warp; v < pieces; v += kWarps) {
        const float *from = part + ((long long)v * 2 + (v > 0)) * a.cols + c0 + lane;
#pragma unroll
        for (int i = 0; i < kJoinCols / 32; ++i)
          if (c0 + i * 32 + lane < a.cols) s[i] += from[i * 32];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kJoinCols / 32; ++i) sm[warp][i * 32 + lane] = s[i];
      __syncthreads();
      const int c = c0 + threadIdx.x;
      if (c < a.cols) {
        float t = 0.0f;
#pragma unroll
        for (int q = 0; q < kWarps; ++q) t += sm[q][threadIdx.x];
        G *out = static_cast<G *>(a.dtable) + w * a.worker_stride + k * a.row_stride + c;
        *out = cdg_cast<G>(a.accumulate ? fmaf(t, a.scale, cdg_ld(out)) : t * a.scale);
      }
    }
  }
}

// m * rows * length below 2^31, without overflow
bool tokens_fit(long long m, long long groups, long long length) {
  constexpr long long most = (1ll << 31) - 1;
  if (groups < 0 || length < 0 || m < 1) return false;
  if (groups == 0 || length == 0) return true;
  return groups <= most / length && groups * length <= most / m;
}

constexpr int kMaxCols = 1 << 24;       // columns are counted in 32 bits, in steps of up to 2^24

constexpr int kSms = 148;

inline long long up16(long long v) { return (v + 15) & ~15ll; }

}  // namespace

extern "C" int cdgrab_embedding_forward(long long groups, long long length, int cols, int vocab, int token_bits, const void *tokens,
                                        long long token_stride, long long padding, float scale, int dtype, const void *table,
                                        long long table_stride, int out_dtype, void *y, long long y_stride, void *stream) {
  if (!tokens_fit(1, groups, length) || cols < 1 || cols > kMaxCols || vocab < 1 || (token_bits != 32 && token_bits != 64) || !std::isfinite(scale) ||
      !cdg_dtype_ok(dtype) || !cdg_dtype_ok(out_dtype))
    return CDGRAB_ERR_INVALID;
  if (groups == 0 || length == 0) return CDGRAB_OK;
  const int e = cdg_dtype_size(dtype), oe = cdg_dtype_size(out_dtype);
  if (!tokens || !table || !y || (groups > 1 && token_stride < length) || (vocab > 1 && table_stride < cols) || y_stride < cols ||
      !cdg_aligned(tokens, token_bits / 8) || !cdg_aligned(table, e) || !cdg_aligned(y, oe))
    return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  const long long rows = groups * length;
  const Tokens tok = {tokens, token_bits, token_stride, length, padding, vocab};
  const int vec = cdg_widest(cols, {{table, vocab > 1 ? table_stride : 0, e}, {y, rows > 1 ? y_stride : 0, oe}});
  const int per_row = cols / vec;
  // One row after another, and a store of eight values everywhere: for short rows, which leave lanes idle row by row.  (2 million bf16
  // values in rows of 37, 106, 257, 515 and 650: 10.1, 8.5, 9.8, 9.4 and 7.7 us, row by row 25.5, 8.6, 12.6, 9.6 and 6.0; of 108 and
  // 260, four values to an access, 7.9 and 7.4, row by row 5.8 and 7.9.)
  const bool flat = vec < 8 && cols >= 8 && cols <= (vec < 4 ? 320 : 64) && (rows == 1 || y_stride == cols) && cdg_aligned(y, 8 * oe);
  const int lv = cdg_widest(cols, {{table, vocab > 1 ? table_stride : 0, e}});
  // four accesses to a lane, but eight lanes where a row has work for them
  int group = 1;
  while (group < 32 && (4 * group < per_row || (group < 8 && group < per_row))) group *= 2;
  const long long blocks = flat ? (rows * cols + 8 * kThreads - 1) / (8 * kThreads) : (rows + kThreads / group - 1) / (kThreads / group);
  if (blocks >= (1ll << 31)) return CDGRAB_ERR_INVALID;
  cudaStream_t st = (cudaStream_t)stream;
  return cdg_by_types(dtype, out_dtype, [&](auto t, auto r) {
    using T = decltype(t);
    using R = decltype(r);
    auto go = [&](auto *kernel) {
      return cdg_launch_rc(cdg_ops_launch(kernel, dim3((unsigned)blocks), kThreads, 0, st, (uint32_t)rows, per_row, group,
                                          cdg_divisor((uint32_t)length), tok, scale, (const T *)table, table_stride, (R *)y, y_stride,
                                          dev->status));
    };
    auto go_flat = [&](auto *kernel) {
      return cdg_launch_rc(cdg_ops_launch(kernel, dim3((unsigned)blocks), kThreads, 0, st, (uint32_t)rows, cdg_divisor((uint32_t)cols),
                                          cdg_divisor((uint32_t)length), tok, scale, (const T *)table, table_stride, (R *)y, dev->status));
    };
    if (flat) return lv >= 4 ? go_flat(lookup_flat_kernel<T, R, 4>) : lv == 2 ? go_flat(lookup_flat_kernel<T, R, 2>) : go_flat(lookup_flat_kernel<T, R, 1>);
    return vec == 8 ? go(lookup_kernel<T, R, 8>) : vec == 4 ? go(lookup_kernel<T, R, 4>) : vec == 2 ? go(lookup_kernel<T, R, 2>)
                                                                                        : go(lookup_kernel<T, R, 1>);
  });
}

extern "C" long long cdgrab_embedding_workspace_bytes(int m, long long tokens, int cols, int vocab) {
  if (m < 1 || m > 65535 || cols < 1 || cols > kMaxCols || vocab < 1 || !tokens_fit(m, 1, tokens)) return -1;
  // the items twice, two sums for each window
  return 2 * up16(8ll * m * tokens) + 8ll * m * ((tokens + kWindow - 1) / kWindow) * cols + 16;
}

extern "C" int cdgrab_embedding_backward(int m, long long groups, long long length, int cols, int vocab, int token_bits,
                                         const void *tokens, long long token_stride, long long padding, float scale, int dtype,
                                         const void *dy, long long dy_stride, int grad_dtype, void *dtable, long long worker_stride,
                                         long long row_stride, int accumulate, void *workspace, long long workspace_bytes,
                                         void *stream) {
  if (m < 1 || m > 65535 || !tokens_fit(m, groups, length)) return CDGRAB_ERR_INVALID;
  const long long n = groups * length, need = cdgrab_embedding_workspace_bytes(m, n, cols, vocab);
  if (need < 0 || (token_bits != 32 && token_bits != 64) || !std::isfinite(scale) || !cdg_dtype_ok(dtype) || !cdg_dtype_ok(grad_dtype) ||
      (accumulate != 0 && accumulate != 1))
    return CDGRAB_ERR_INVALID;
  if (accumulate && n == 0) return CDGRAB_OK;
  const int e = cdg_dtype_size(dtype), ge = cdg_dtype_size(grad_dtype);
  if (!dtable || (vocab > 1 && (row_stride < cols || row_stride > (1ll << 32))) ||
      (m > 1 && (worker_stride < (vocab - 1) * row_stride + cols || worker_stride > (1ll << 46))) || !cdg_aligned(dtable, ge))
    return CDGRAB_ERR_INVALID;
  if (n > 0 && (!tokens || !dy || (m * groups > 1 && token_stride < length) || (m * n > 1 && dy_stride < cols) ||
                !cdg_aligned(tokens, token_bits / 8) || !cdg_aligned(dy, e)))
    return CDGRAB_ERR_INVALID;
  if (!workspace || workspace_bytes < need || !cdg_aligned(workspace, 16)) return CDGRAB_ERR_INVALID;
  const CdgOpsDevice *dev;
  if (const int rc = cdg_ops_device(&dev)) return rc;
  cudaStream_t st = (cudaStream_t)stream;

  Sort s = {};
  s.tok = {tokens, token_bits, token_stride, length, padding, vocab};
  s.length = cdg_divisor((uint32_t)(n > 0 ? length : 1));
  s.groups = (int)groups;
  s.n = (int)n;
  int key_bits = 1;
  while (key_bits < 31 && (vocab >> key_bits) > 0) ++key_bits;       // of the number behind the vocabulary
  s.passes = (key_bits + 7) / 8;
  s.bits = (key_bits + s.passes - 1) / s.passes;
  s.items = static_cast<uint2 *>(workspace);
  s.other = reinterpret_cast<uint2 *>(static_cast<uint8_t *>(workspace) + up16(8 * m * n));
  s.status = dev->status;
  // a CTA for every kShare of a worker's tokens, up to eight, while there are SMs for them
  int ctas = 1;
  while (ctas < 8 && n > kShare * ctas && 2ll * ctas * m <= dev->sms) ctas *= 2;
  const unsigned sorting = n > 0 ? (unsigned)(m * ctas) : 0;
  Clear z = {};
  if (!accumulate) {
    z.p = dtable;
    z.elem = ge;
    z.worker_stride = worker_stride;
    z.row_stride = vocab > 1 ? row_stride : cols;
    z.cols = cols;
    z.vocab = vocab;
    z.rows_per_block = 131072 / ((long long)cols * ge);
    if (z.rows_per_block < 1) z.rows_per_block = 1;
    z.blocks_per_worker = (vocab + z.rows_per_block - 1) / z.rows_per_block;
    z.blocks = m * z.blocks_per_worker;
  }
  const long long clearing = z.blocks < (1ll << 24) ? (z.blocks + ctas - 1) / ctas * ctas : 1ll << 24;
  if (const int rc = tc_launch_cluster(sort_and_clear_kernel, dim3((unsigned)(sorting + clearing)), ctas, kSortThreads, 0, st, s, z, sorting)) return rc;
  if (n == 0) return CDGRAB_OK;

  Sums a = {s.items, (int)n, (int)((n + kWindow - 1) / kWindow), vocab, cols, nullptr, dy, dy_stride, dtable, worker_stride, row_stride, scale,
            accumulate};
  a.part = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + 2 * up16(8 * m * n));
  const long long all = (long long)m * a.windows;
  const int vec = cdg_widest(cols, {{dy, m * n > 1 ? dy_stride : 0, e}, {dtable, vocab > 1 ? row_stride : 0, ge}, {dtable, m > 1 ? worker_stride : 0, ge}});
  // up to eight values, four accesses or 16 bytes to a lane, as many as the columns need.  (32 x 700 rows of 650 fp32: 144 us, with 32 bytes 165: too
  // few warps)  And no more than leave 32 warps to an SM.
  int nv = 1;
  while (vec * nv < 8 && nv < 4 && vec * nv * e < 16 && 32 * vec * nv < cols && all * cols > 32ll * vec * nv * 32 * kSms) nv *= 2;
  auto slabs = [&](int width) { return (unsigned)((cols + width - 1) / width < 65535 ? (cols + width - 1) / width : 65535); };
  const int rc = cdg_by_types(dtype, grad_dtype, [&](auto t, auto g) {
    using T = decltype(t);
    using G = decltype(g);
    auto go = [&](auto *kernel) {
      return cdg_launch_rc(cdg_ops_launch(kernel, dim3((unsigned)((all + kSumThreads / 32 - 1) / (kSumThreads / 32)), slabs(32 * vec * nv)), kSumThreads, 0, st, a, all));
    };
    if constexpr (sizeof(T) == 2) {          // (of fp32 they would be 32 bytes to a lane)
      if (vec == 4 && nv == 2) return go(run_sums_kernel<T, G, 4, 2>);
      if (vec == 2 && nv == 4) return go(run_sums_kernel<T, G, 2, 4>);
    }
    switch (vec * 10 + nv) {
      case 81: return go(run_sums_kernel<T, G, 8, 1>);
      case 41: return go(run_sums_kernel<T, G, 4, 1>);
      case 21: return go(run_sums_kernel<T, G, 2, 1>);
      case 22: return go(run_sums_kernel<T, G, 2, 2>);
      case 11: return go(run_sums_kernel<T, G, 1, 1>);
      case 12: return go(run_sums_kernel<T, G, 1, 2>);
      default: return go(run_sums_kernel<T, G, 1, 4>);
    }
  });
  if (rc != CDGRAB_OK || n <= 2 * kWindow) return rc;         // no run goes on past two windows
  const dim3 grid((unsigned)((all + kJoin - 1) / kJoin), slabs(kJoinCols));
  return cdg_launch_rc(grad_dtype == CDGRAB_F32 ? cdg_ops_launch(join_runs_kernel<float>, grid, kThreads, 0, st, a, all)
                                                : cdg_ops_launch(join_runs_kernel<__nv_bfloat16>, grid, kThreads, 0, st, a, all));
}
