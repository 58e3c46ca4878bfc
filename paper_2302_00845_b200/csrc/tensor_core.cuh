// Helpers of the operators' tcgen05 kernels: tensor memory, matrix instructions, tensor maps.
#pragma once

#include "operators.cuh"
#include "ptx.cuh"

// ---- shared-memory operand tiles --------------------------------------------------------------
// A tile is a column of panels; a panel holds 64 16-bit values of each row, rows 128 bytes apart,
// with the 128-byte swizzle the bulk copies write (its 8-row groups start on 1024-byte boundaries).
//
// K-major: the rows are the operand's M (or N) index and the 64 columns its K index.  Eight rows
// are 1024 bytes; 16 values of K are 32 bytes further on inside the same rows.
__device__ __forceinline__ uint64_t tc_desc_k(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}
// MN-major: the rows are the K index and the columns the M (or N) index.  Eight values of K are
// 1024 bytes (the stride offset); 64 further values of M or N are the next panel (the leading
// offset, `panel` bytes); 16 values of K are 2048 bytes further on.
__device__ __forceinline__ uint64_t tc_desc_mn(uint32_t saddr, uint32_t panel) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(panel >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// instruction descriptor of kind::f16: fp32 accumulator, A and B of one type, N columns, M rows
__host__ __device__ constexpr uint32_t tc_idesc(bool bf16, int m, int n, bool a_mn, bool b_mn) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) |
         ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// true in one lane of a converged warp, the same one every time
__device__ __forceinline__ bool tc_elect() {
  uint32_t pred;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(pred));
  return pred != 0;
}

// D (tensor memory) = A B (+ D), A and B in shared memory; issued by one thread
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// ... with A in tensor memory: lane = row, two 16-bit values of K to a 32-bit column
__device__ __forceinline__ void tc_mma_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// the barrier completes when the matrix instructions issued so far by this thread have
__device__ __forceinline__ void tc_commit(uint64_t *bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// bounded wait of a whole warp, whose lanes stay together; false when it expired
__device__ __forceinline__ bool tc_wait(uint64_t *bar, uint32_t parity, long long deadline) {
  while (true) {
    uint32_t done;
    asm volatile(
        "{\n.reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n}"
        : "=r"(done) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    if (__all_sync(0xffffffffu, done)) return true;
    if (__any_sync(0xffffffffu, clock64() > deadline)) return false;
  }
}
// The matrix instructions that this warp has issued are over.  At a kernel's end, before the tensor memory and the tiles
// that they use are given up: where another role's wait has expired nobody else has waited for them.  `bar`: initialised
// with one arrival, used for nothing else.
__device__ __forceinline__ void tc_finish(uint64_t *bar) {
  __syncwarp();
  if (tc_elect()) tc_commit(bar);
  __syncwarp();
  tc_wait(bar, 0, clock64() + kCdgWaitCycles);
}
// tile from shared memory to a tensor (one thread; coordinates inside the tensor); the end of a group of such
// copies, and waits for this thread's groups: all but the last to have read shared memory, all to be written
__device__ __forceinline__ void tc_store_3d(const CUtensorMap *map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tc_store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void tc_store_read1() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }
__device__ __forceinline__ void tc_store_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// moves registers between warpgroups: all four warps of one execute it.  The shares have to add up to
// no more than the block was launched with.
template <int N> __device__ __forceinline__ void tc_regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void tc_regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// ---- tensor memory ----------------------------------------------------------------------------
// one whole warp; `columns` a power of two from 32
__device__ __forceinline__ void tc_alloc(uint32_t *slot, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tc_free(uint32_t base, uint32_t columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// generic writes to shared memory become visible to bulk copies and matrix instructions
__device__ __forceinline__ void tc_proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 32 columns of this warp's 32 lanes: thread t gets lane t, one value per column
__device__ __forceinline__ void tc_load32(uint32_t addr, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]),
        "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
        "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(addr));
}
__device__ __forceinline__ void tc_store32(uint32_t addr, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]),
        "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]),
        "r"(v[30]), "r"(v[31]) : "memory");
}

// ---- rings, persistent CTAs, clusters -------------------------------------------------------------
// Turn n of a ring of R stages uses stage n % R in the phase of tc_parity(n, R); counters run on over a
// persistent CTA's blocks.
__device__ __forceinline__ uint32_t tc_parity(int n, int ring) { return (uint32_t)(n / ring) & 1u; }
// waits for the stage of turn n to have been released by turn n - ring (one thread)
__device__ __forceinline__ bool tc_wait_released(uint64_t *empty, int n, int ring, long long deadline) {
  return n < ring || mbar_wait(smem_u32(&empty[n % ring]), tc_parity(n - ring, ring), deadline);
}
// the last copies of a ring have to land before the CTA gives up its shared memory (where a wait has expired, nobody
// else has waited for them)
__device__ __forceinline__ void tc_drain(uint64_t *full, int n, int ring) {
  for (int i = max(0, n - ring); i < n; ++i) mbar_wait(smem_u32(&full[i % ring]), tc_parity(i, ring), clock64() + kCdgWaitCycles);
}
// Cluster launch control: a CTA that has finished its block takes over the next CTA of the grid that has
// not been started.  One answer is fetched ahead; `readers` warps (or single threads) follow it.
struct TcQueue { uint4 answer[2]; uint64_t full[2], empty[2]; };       // in shared memory: the next block, one ahead
__device__ __forceinline__ void tc_queue_init(TcQueue &q, int readers) {
  for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&q.full[i]), 1); mbar_init(smem_u32(&q.empty[i]), readers); }
}
// asks for block number `seq` of this CTA (one thread)
__device__ __forceinline__ bool tc_queue_ask(TcQueue &q, int seq, long long deadline) {
  const int s = seq & 1;
  if (!tc_wait_released(q.empty, seq, 2, deadline)) return false;
  mbar_expect_tx(smem_u32(&q.full[s]), 16);
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
               ::"r"(smem_u32(&q.answer[s])), "r"(smem_u32(&q.full[s])) : "memory");
  return true;
}
// ... and reads the answer: the block, or -1 when none is left
__device__ __forceinline__ long long tc_queue_answer(TcQueue &q, int seq) {
  uint32_t got, x;
  asm volatile(
      "{\n.reg .b128 h;\n.reg .pred p;\nld.shared.b128 h, [%2];\n"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\nselp.u32 %0, 1, 0, p;\nmov.u32 %1, 0;\n"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, _, _, _}, h;\n}"
      : "=r"(got), "=r"(x) : "r"(smem_u32(&q.answer[seq & 1])) : "memory");
  tc_proxy_fence();              // the next answer may be written once this one has been read
  return got ? (long long)x : -1;
}
__device__ __forceinline__ long long tc_queue_next(TcQueue &q, int seq, long long deadline, bool &ok) {        // a whole warp
  if (!(ok = ok && tc_wait(&q.full[seq & 1], tc_parity(seq, 2), deadline))) return -1;
  const long long at = tc_queue_answer(q, seq);
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&q.empty[seq & 1]));
  return at;
}
__device__ __forceinline__ long long tc_queue_next_one(TcQueue &q, int seq, long long deadline, bool &ok) {    // one thread
  if (!(ok = ok && mbar_wait(smem_u32(&q.full[seq & 1]), tc_parity(seq, 2), deadline))) return -1;
  const long long at = tc_queue_answer(q, seq);
  mbar_arrive(smem_u32(&q.empty[seq & 1]));
  return at;
}
__device__ __forceinline__ void tc_warp_arrive(uint64_t *bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(bar));
}

__device__ __forceinline__ uint32_t tc_cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t tc_cluster_size() { uint32_t r; asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void tc_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// arrives at the barrier of another CTA of the cluster, and waits for such arrivals (a whole warp)
__device__ __forceinline__ void tc_arrive_peer(uint64_t *bar, uint32_t rank) {
  asm volatile("{\n.reg .b32 there;\nmapa.shared::cluster.u32 there, %0, %1;\n"
               "mbarrier.arrive.release.cluster.shared::cluster.b64 _, [there];\n}" ::"r"(smem_u32(bar)), "r"(rank) : "memory");
}
__device__ __forceinline__ bool tc_wait_cluster(uint64_t *bar, uint32_t parity, long long deadline) {
  uint32_t done;
  while (true) {
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
        : "=r"(done) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    if (done || clock64() > deadline) break;
  }
  return __all_sync(0xffffffffu, done != 0);
}
// 16 bytes of another CTA's shared memory
__device__ __forceinline__ float4 tc_peer_load(uint32_t addr, uint32_t rank) {
  uint32_t there;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(there) : "memory");
  return v;
}

// ---- host side ----------------------------------------------------------------------------------
// Tensor map of 16-bit values: dims / strides[i] (elements; the innermost axis is contiguous), box of
// 64 columns by `box_rows` rows with the 128-byte swizzle (or of 32 columns with the 64-byte one);
// out-of-range elements read as zeros and are not written.
inline bool tc_encode(CUtensorMap *map, bool bf16, const void *base, int rank, const long long *dims,
                      const long long *strides, int box_rows, int box_cols = 64) {
  typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                               const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                               CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  EncodeFn fn = (EncodeFn)cdg_tensor_map_encoder();
  if (!fn) return false;
  cuuint64_t d[5], s[4];
  cuuint32_t box[5], one[5];
  for (int i = 0; i < rank; ++i) {
    d[i] = (cuuint64_t)dims[i];
    if (i > 0) s[i - 1] = (cuuint64_t)strides[i] * 2;
    box[i] = i == 0 ? (cuuint32_t)box_cols : i == 1 ? (cuuint32_t)box_rows : 1;
    one[i] = 1;
  }
  return fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank,
            const_cast<void *>(base), d, s, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename... KArgs, typename... Args>
inline int tc_launch_cluster(void (*kernel)(KArgs...), dim3 grid, int cluster, int threads, size_t smem, cudaStream_t st, Args... args) {
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

template <typename K>
inline bool tc_raise_limit(CdgPerDevice &flags, K *kernel, size_t bytes) {
  int dev = 0;
  return cudaGetDevice(&dev) == cudaSuccess && cdg_raise_smem_limit(flags, dev, kernel, bytes) == cudaSuccess;
}

