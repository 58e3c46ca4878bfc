// Rows of fp32 or bf16 values moved several to an access: what embedding, dropout and the rotation share.
#pragma once

#include <initializer_list>

#include "operators.cuh"

inline bool cdg_dtype_ok(int t) { return t == CDGRAB_F32 || t == CDGRAB_BF16; }
inline int cdg_dtype_size(int t) { return t == CDGRAB_F32 ? 4 : 2; }

// A tensor of rows as an operator reads or writes it: address, distance of the rows in elements, type.
struct CdgRows {
  const void *p;
  long long stride;
  int elem;        // bytes
};
// The most values (8, 4, 2 or 1) to an access that the row length and every tensor's address and stride allow: an access of
// n values starts at a multiple of n values and of their bytes, 32 at most.
inline int cdg_widest(long long cols, std::initializer_list<CdgRows> tensors) {
  for (int n : {8, 4, 2}) {
    bool ok = cols % n == 0;
    for (const CdgRows &t : tensors) ok = ok && (!t.p || (t.stride % n == 0 && cdg_aligned(t.p, n * t.elem)));
    if (ok) return n;
  }
  return 1;
}

// Division of numbers below 2^31 by a fixed one (Granlund and Montgomery, 1994).
struct CdgDivisor {
  uint32_t d, mul, shift;
};
inline CdgDivisor cdg_divisor(uint32_t d) {
  uint32_t shift = 0;
  while (shift < 32 && (1ull << shift) < d) ++shift;
  return {d, (uint32_t)((((1ull << shift) - d) << 32) / d + 1), shift};
}

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t cdg_divide(uint32_t n, const CdgDivisor &v) { return (__umulhi(n, v.mul) + n) >> v.shift; }

// N adjacent values of type T in registers, as they lie in memory
template <typename T, int N>
struct CdgVec {
  static constexpr int kBytes = N * (int)sizeof(T), kWords = kBytes < 4 ? 1 : kBytes / 4;
  uint32_t w[kWords];

  __device__ __forceinline__ void load(const T *p) {
    if constexpr (kBytes == 32)
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
    else if constexpr (kBytes == 16)
      asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
    else if constexpr (kBytes == 8)
      asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
    else if constexpr (kBytes == 4)
      asm volatile("ld.global.b32 %0, [%1];" : "=r"(w[0]) : "l"(p));
    else
      asm volatile("ld.global.u16 %0, [%1];" : "=r"(w[0]) : "l"(p));
  }
  // What p points to, or what was there before: one instruction under a predicate, no branch.
  __device__ __forceinline__ void load_if(bool yes, const T *p) {
    const int go = yes;
    if constexpr (kBytes == 32)
      asm volatile("{\n.reg .pred q;\nsetp.ne.s32 q, %9, 0;\n@q ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n}"
                   : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3]), "+r"(w[4]), "+r"(w[5]), "+r"(w[6]), "+r"(w[7]) : "l"(p), "r"(go));
    else if constexpr (kBytes == 16)
      asm volatile("{\n.reg .pred q;\nsetp.ne.s32 q, %5, 0;\n@q ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n}"
                   : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3]) : "l"(p), "r"(go));
    else if constexpr (kBytes == 8)
      asm volatile("{\n.reg .pred q;\nsetp.ne.s32 q, %3, 0;\n@q ld.global.v2.b32 {%0, %1}, [%2];\n}" : "+r"(w[0]), "+r"(w[1]) : "l"(p), "r"(go));
    else if constexpr (kBytes == 4)
      asm volatile("{\n.reg .pred q;\nsetp.ne.s32 q, %2, 0;\n@q ld.global.b32 %0, [%1];\n}" : "+r"(w[0]) : "l"(p), "r"(go));
    else
      asm volatile("{\n.reg .pred q;\nsetp.ne.s32 q, %2, 0;\n@q ld.global.u16 %0, [%1];\n}" : "+r"(w[0]) : "l"(p), "r"(go));
  }
  __device__ __forceinline__ void store(T *p) const { store_if(true, p); }
  __device__ __forceinline__ void store_if(bool yes, T *p) const {
    const int go = yes;
    if constexpr (kBytes == 32)
      asm volatile("{\n.reg .pred q;\nsetp.ne.s32 q, %9, 0;\n@q st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};\n}"
                   ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "l"(p), "r"(go) : "memory");
    else if constexpr (kBytes == 16)
      asm volatile("{\n.reg .pred q;\nsetp.ne.s32 q, %5, 0;\n@q st.global.v4.b32 [%4], {%0, %1, %2, %3};\n}"
                   ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "l"(p), "r"(go) : "memory");
    else if constexpr (kBytes == 8)
      asm volatile("{\n.reg .pred q;\nsetp.ne.s32 q, %3, 0;\n@q st.global.v2.b32 [%2], {%0, %1};\n}" ::"r"(w[0]), "r"(w[1]), "l"(p), "r"(go) : "memory");
    else if constexpr (kBytes == 4)
      asm volatile("{\n.reg .pred q;\nsetp.ne.s32 q, %2, 0;\n@q st.global.b32 [%1], %0;\n}" ::"r"(w[0]), "l"(p), "r"(go) : "memory");
    else
      asm volatile("{\n.reg .pred q;\nsetp.ne.s32 q, %2, 0;\n@q st.global.u16 [%1], %0;\n}" ::"r"(w[0]), "l"(p), "r"(go) : "memory");
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0u;
  }
  __device__ __forceinline__ float get(int i) const {       // i known at compile time
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  // all values, each rounded once
  __device__ __forceinline__ void set(const float (&f)[N]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = __float_as_uint(f[i]);
    } else if constexpr (N == 1) {
      w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(f[0]));
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(f[i], f[(i + 1) % N]);
        w[i / 2] = *reinterpret_cast<const uint32_t *>(&v);
      }
    }
  }
};

// f(T(), R()) for the types that two codes name
template <typename F>
inline int cdg_by_types(int a, int b, F &&f) {
  if (a == CDGRAB_F32) return b == CDGRAB_F32 ? f(0.0f, 0.0f) : f(0.0f, __nv_bfloat16());
  return b == CDGRAB_F32 ? f(__nv_bfloat16(), 0.0f) : f(__nv_bfloat16(), __nv_bfloat16());
}
#endif
