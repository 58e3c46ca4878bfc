// Philox4x32-10 (Salmon et al., SC 2011), the counter-based generator of the seeded draws and of dropout.
#pragma once

#include <stdint.h>

// what the two key words grow by from round to round
constexpr uint32_t kPhiloxWeyl0 = 0x9E3779B9u, kPhiloxWeyl1 = 0xBB67AE85u;

// A round:  (c0, c1, c2, c3) <- (hi(M1 c2) ^ c1 ^ k0, lo(M1 c2), hi(M0 c0) ^ c3 ^ k1, lo(M0 c0)).
__host__ __device__ inline void cdg_philox_round(uint32_t &c0, uint32_t &c1, uint32_t &c2, uint32_t &c3, uint32_t k0, uint32_t k1) {
  const unsigned long long p0 = 0xD2511F53ull * c0, p1 = 0xCD9E8D57ull * c2;
  const uint32_t n0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0, n2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
  c1 = (uint32_t)p1; c3 = (uint32_t)p0; c0 = n0; c2 = n2;
}
// ten of them
__host__ __device__ inline void cdg_philox4x32_10(uint32_t &c0, uint32_t &c1, uint32_t &c2, uint32_t &c3, uint32_t k0,
                                                  uint32_t k1) {
#pragma unroll
  for (int round = 0; round < 10; ++round)
    cdg_philox_round(c0, c1, c2, c3, k0 + round * kPhiloxWeyl0, k1 + round * kPhiloxWeyl1);
}
