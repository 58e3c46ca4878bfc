// Embedding lookup and its gradient, reduced per worker into the gather buffer.
//
//   y[r] = scale table[t_r];   dtable[i][v] = scale sum of dy[r] over worker i's rows r with t_r = v.
//
// The lookup is bound by memory: a row read (from L2 where tokens repeat) and a row written.  The gradient writes every row of
// every worker's table, most of them zero, and reads dy once.  It runs in three launches:
//   1. each worker's tokens are sorted by value, stably, by a cluster of its own, while the other blocks clear the tables;
//   2. runs of equal tokens are summed in the order of their positions, a warp to 32 sorted positions and 256 columns;
//   3. runs that go on over more than two such windows, which step 2 leaves as a sum for each window, are joined in order.
// No sum depends on the order in which blocks run, and nothing is added to memory by atomics.
#include <cmath>

#include "rows.cuh"
#include "tensor_core.cuh"

#ifndef AH
#define AH 8
#endif
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
      if (valid && c + u * group < per_row) v[u].load(from + u * step);
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
#ifndef KSH
#define KSH 1024
#endif
constexpr long long kShare = KSH;     // items to a CTA while more CTAs can be had

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

#ifndef SMB
#define SMB 2
#endif
__global__ void __launch_bounds__(kSortThreads, SMB) sort_and_clear_kernel(const __grid_constant__ Sort s, const __grid_constant__ Clear z,
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
// A window is 32 sorted positions.  A run that starts in window w and ends in it or in the next one belongs to w, which sums all of it.
// A longer one is summed window by window: its part in the window it starts in goes to part[w][0], its parts in the windows it
// goes on in to part[.][1].  Keys 33 positions back and 64 ahead tell which case it is, without a search.
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
constexpr int kSlab = 256;             // columns to a warp, eight to a lane

template <typename T, typename G, int VEC>
__global__ void __launch_bounds__(kThreads) run_sums_kernel(const __grid_constant__ Sums a, long long all) {
  constexpr int NV = 8 / VEC, kAhead = AH;
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int lane = threadIdx.x & 31;
  const long long at = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);      // worker and window
  if (at >= all) return;
  const long long w = at / a.windows;
  const int p0 = (int)(at - w * a.windows) * 32;
  const uint2 *items = a.items + w * a.n;
  auto key = [&](long long p) { return p >= 0 && p < a.n ? items[p].x : kNoKey; };
  uint2 e[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) e[k] = (long long)p0 + 32 * k + lane < a.n ? items[p0 + 32 * k + lane] : make_uint2(kNoKey, 0u);
  const uint32_t back1 = key((long long)p0 - 1), back33 = key((long long)p0 - 33), ahead = key((long long)p0 + 64);
  const uint32_t first = __shfl_sync(0xffffffffu, e[0].x, 0), last = __shfl_sync(0xffffffffu, e[0].x, 31);
  const uint32_t next = __shfl_sync(0xffffffffu, e[1].x, 0);
  // tokens without a gradient are past the others, and what is past the end behind them
  const int live = __popc(__ballot_sync(0xffffffffu, e[0].x < (uint32_t)a.vocab));
  if (live == 0) return;
  const bool goes_on = first == back1;                                  // the first run began before
  const bool head_long = goes_on && (first == back33 || first == next);
  const int head = __popc(__ballot_sync(0xffffffffu, e[0].x == first)); // its positions here
  const bool whole = head == 32 && goes_on;                             // nothing begins here
  const bool tail_long = !whole && live == 32 && last == ahead;
  int begin = goes_on && !head_long ? head : 0, end = live;
  if (!whole && live == 32 && !tail_long) end += __popc(__ballot_sync(0xffffffffu, e[1].x == last));
  if (begin >= end) return;
  const long long rows = w * a.n;
  for (int c0 = blockIdx.y * kSlab; c0 < a.cols; c0 += gridDim.y * kSlab) {
    float acc[NV][VEC] = {};
    const T *dy = static_cast<const T *>(a.dy) + c0 + lane * VEC;
    auto flush = [&](uint32_t k, float *part) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = c0 + (i * 32 + lane) * VEC;
        if (c < a.cols) {
          if (part) {
#pragma unroll
            for (int f = 0; f < VEC; ++f) part[c + f] = acc[i][f];
          } else {
            G *out = static_cast<G *>(a.dtable) + w * a.worker_stride + k * a.row_stride + c;
            CdgVec<G, VEC> o;
            float v[VEC];
            if (a.accumulate) o.load(out);
#pragma unroll
            for (int f = 0; f < VEC; ++f) v[f] = a.accumulate ? fmaf(acc[i][f], a.scale, o.get(f)) : acc[i][f] * a.scale;
            o.set(v);
            o.store(out);
          }
        }
#pragma unroll
        for (int f = 0; f < VEC; ++f) acc[i][f] = 0.0f;
      }
    };
    float *part = a.part + ((w * a.windows + p0 / 32) * 2) * (long long)a.cols;
    for (int p = begin; p < end; p += kAhead) {
      CdgVec<T, VEC> v[kAhead][NV];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int q = min(p + u, end - 1);
        const uint32_t r0 = __shfl_sync(0xffffffffu, e[0].y, q & 31), r1 = __shfl_sync(0xffffffffu, e[1].y, q & 31);
        const T *row = dy + (rows + (q < 32 ? r0 : r1)) * a.dy_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (c0 + (i * 32 + lane) * VEC < a.cols) v[u][i].load(row + i * 32 * VEC);
          else v[u][i].zero();
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int q = p + u;
        if (q >= end) break;
        const uint32_t k0 = __shfl_sync(0xffffffffu, e[0].x, q & 31), k1 = __shfl_sync(0xffffffffu, e[1].x, q & 31);
        const uint32_t n0 = __shfl_sync(0xffffffffu, e[0].x, (q + 1) & 31), n1 = __shfl_sync(0xffffffffu, e[1].x, (q + 1) & 31);
        const uint32_t k = q < 32 ? k0 : k1;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int f = 0; f < VEC; ++f) acc[i][f] += v[u][i].get(f);
        if (q + 1 == end || k != (q + 1 < 32 ? n0 : n1)) {
          const bool is_head = goes_on && q + 1 == head;
          flush(k, is_head ? part + a.cols : tail_long && q + 1 == end ? part : nullptr);
        }
      }
    }
  }
}

// a block to kJoin windows and 256 columns: the parts of each long run that starts there, warp q taking every eighth
constexpr int kJoin = 8;
template <typename G>
__global__ void __launch_bounds__(kThreads) join_runs_kernel(const __grid_constant__ Sums a, long long all) {
  __shared__ float sm[kWarps][kSlab];
  cdg_grid_dep_wait();
  cdg_grid_dep_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int j = 0; j < kJoin; ++j) {
    const long long at = (long long)blockIdx.x * kJoin + j;
    if (at >= all) return;
    const long long w = at / a.windows;
    const int win = (int)(at - w * a.windows), p0 = win * 32;
    const uint2 *items = a.items + w * a.n;
    if ((long long)p0 + 64 >= a.n) continue;
    const uint32_t k = items[p0 + 31].x;
    if (k >= (uint32_t)a.vocab || items[p0 + 64].x != k || (p0 > 0 && items[p0 - 1].x == k)) continue;
    for (int c0 = blockIdx.y * kSlab; c0 < a.cols; c0 += gridDim.y * kSlab) {
      const float *part = a.part + (w * a.windows + win) * 2 * (long long)a.cols;
      float s[kSlab / 32] = {};
      for (int v = win + warp; v < a.windows && items[(long long)v * 32 + (v == win ? 31 : 0)].x == k; v += kWarps) {
        const float *from = part + ((long long)(v - win) * 2 + (v == win ? 0 : 1)) * a.cols;
#pragma unroll
        for (int i = 0; i < kSlab / 32; ++i) {
          const int c = c0 + i * 32 + lane;
          if (c < a.cols) s[i] += from[c];
        }
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kSlab / 32; ++i) sm[warp][i * 32 + lane] = s[i];
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

inline long long up16(long long v) { return (v + 15) & ~15ll; }

}  // namespace

extern "C" int cdgrab_embedding_forward(long long groups, long long length, int cols, int vocab, int token_bits, const void *tokens,
                                        long long token_stride, long long padding, float scale, int dtype, const void *table,
                                        long long table_stride, int out_dtype, void *y, long long y_stride, void *stream) {
  if (!tokens_fit(1, groups, length) || cols < 1 || vocab < 1 || (token_bits != 32 && token_bits != 64) || !std::isfinite(scale) ||
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
  // four accesses to a lane, but eight lanes where a row has work for them
  int group = 1;
  while (group < 32 && (4 * group < per_row || (group < 8 && group < per_row))) group *= 2;
  const long long blocks = (rows + kThreads / group - 1) / (kThreads / group);
  cudaStream_t st = (cudaStream_t)stream;
  return cdg_by_types(dtype, out_dtype, [&](auto t, auto r) {
    using T = decltype(t);
    using R = decltype(r);
    auto go = [&](auto *kernel) {
      return cdg_launch_rc(cdg_ops_launch(kernel, dim3((unsigned)blocks), kThreads, 0, st, (uint32_t)rows, per_row, group,
                                          cdg_divisor((uint32_t)length), tok, scale, (const T *)table, table_stride, (R *)y, y_stride,
                                          dev->status));
    };
    return vec == 8 ? go(lookup_kernel<T, R, 8>) : vec == 4 ? go(lookup_kernel<T, R, 4>) : vec == 2 ? go(lookup_kernel<T, R, 2>)
                                                                                        : go(lookup_kernel<T, R, 1>);
  });
}

extern "C" long long cdgrab_embedding_workspace_bytes(int m, long long tokens, int cols, int vocab) {
  if (m < 1 || m > 65535 || cols < 1 || vocab < 1 || !tokens_fit(m, 1, tokens)) return -1;
  // the items twice, two sums for each window
  return 2 * up16(8ll * m * tokens) + 8ll * m * ((tokens + 31) / 32) * cols + 16;
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

  Sums a = {s.items, (int)n, (int)((n + 31) / 32), vocab, cols, nullptr, dy, dy_stride, dtable, worker_stride, row_stride, scale, accumulate};
  a.part = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + 2 * up16(8 * m * n));
  const long long all = (long long)m * a.windows;
  const unsigned slabs = (unsigned)((cols + kSlab - 1) / kSlab < 65535 ? (cols + kSlab - 1) / kSlab : 65535);
  const int vec = cdg_widest(cols, {{dy, m * n > 1 ? dy_stride : 0, e}, {dtable, vocab > 1 ? row_stride : 0, ge}, {dtable, m > 1 ? worker_stride : 0, ge}});
  const int rc = cdg_by_types(dtype, grad_dtype, [&](auto t, auto g) {
    using T = decltype(t);
    using G = decltype(g);
    auto go = [&](auto *kernel) {
      return cdg_launch_rc(cdg_ops_launch(kernel, dim3((unsigned)((all + kWarps - 1) / kWarps), slabs), kThreads, 0, st, a, all));
    };
    return vec == 8 ? go(run_sums_kernel<T, G, 8>) : vec == 4 ? go(run_sums_kernel<T, G, 4>) : vec == 2 ? go(run_sums_kernel<T, G, 2>)
                                                                                             : go(run_sums_kernel<T, G, 1>);
  });
  if (rc != CDGRAB_OK || n <= 64) return rc;         // no run goes on past two windows
  const dim3 grid((unsigned)((all + kJoin - 1) / kJoin), slabs);
  return cdg_launch_rc(grad_dtype == CDGRAB_F32 ? cdg_ops_launch(join_runs_kernel<float>, grid, kThreads, 0, st, a, all)
                                                : cdg_ops_launch(join_runs_kernel<__nv_bfloat16>, grid, kThreads, 0, st, a, all));
}
