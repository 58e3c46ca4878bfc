// Shared by the training operators (layer norm, attention, orthogonalised update, embedding, dropout, rotation): the device they
// run on, their status word, and small device helpers.
#pragma once

#include "common.cuh"

struct CdgOpsDevice {
  int index;      // the device
  int sms;        // multiprocessors
  int *status;    // the operators' device status word (CDG_ST_* bits)
};
// the current device, looked up once per device; CDGRAB_ERR_DEVICE when it is no sm_100
int cdg_ops_device(const CdgOpsDevice **out);
// how long a device-side wait of the next launches may last, in clock cycles
long long cdg_ops_wait_limit();

inline bool cdg_aligned(const void *p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// Strides (batch, token, head) of a [batch][token][head][dim] tensor that is read: multiples of 8 values, tokens and heads apart
// from each other.
inline bool cdg_heads_in_ok(const long long s[3], int tokens, int heads, int dim, long long most) {
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] % 8 != 0 || s[i] > most) return false;
  return (tokens <= 1 || s[1] >= dim) && (heads <= 1 || s[2] >= dim);
}
// ... and of one that is written: no two heads' values on top of each other
inline bool cdg_heads_out_ok(const long long s[3], int batch, int tokens, int heads, int dim, long long most) {
  if (!cdg_heads_in_ok(s, tokens, heads, dim, most)) return false;
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

// the error of the launches since the last check, as a CDGRAB_* code
inline int cdg_launch_rc(cudaError_t e = cudaSuccess) {
  const cudaError_t l = cudaGetLastError();
  return e == cudaSuccess && l == cudaSuccess ? CDGRAB_OK : CDGRAB_ERR_CUDA;
}

#ifdef __CUDACC__
template <typename T> __device__ __forceinline__ T cdg_cast(float v);
template <> __device__ __forceinline__ float cdg_cast<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 cdg_cast<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ float cdg_warp_sum(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}

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

// Launch that may be scheduled while its predecessor in the stream still runs; every thread of the
// kernel has to call cdg_grid_dep_wait() before it reads or writes global memory.
template <typename... KArgs, typename... Args>
inline cudaError_t cdg_ops_launch(void (*kernel)(KArgs...), dim3 grid, int threads, size_t smem, cudaStream_t st,
                                  Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}
#endif
