// Philox4x32-10, a counter-based random generator: ten rounds of a bijection of
// a 128-bit counter under a 64-bit key (Salmon, Moraes, Dror, Shaw, "Parallel
// random numbers: as easy as 1, 2, 3", SC 2011). Plain arithmetic, for host and
// device.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define ABFT_BOTH __host__ __device__ __forceinline__
#else
#define ABFT_BOTH inline
#endif

namespace abft {

struct Philox {
  uint32_t w[4];
};

ABFT_BOTH uint32_t xor3(uint32_t x, uint32_t y, uint32_t z) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_amdgcn_bitop3_b32(x, y, z, 0x96);  // one instruction; the table of x ^ y ^ z
#else
  return x ^ y ^ z;
#endif
}

ABFT_BOTH Philox philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0,
                        uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p0 = uint64_t(0xD2511F53u) * c0, p1 = uint64_t(0xCD9E8D57u) * c2;
    c0 = xor3(uint32_t(p1 >> 32), c1, k0);
    c2 = xor3(uint32_t(p0 >> 32), c3, k1);
    c1 = uint32_t(p1);
    c3 = uint32_t(p0);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return Philox{{c0, c1, c2, c3}};
}

// Dropout's draws of the elements 8 chunk .. 8 chunk + 7 of a row: 16 bits each,
// the low half of word 0 first. chunk < 2^13, site < 2^16.
ABFT_BOTH Philox dropout_draws(uint64_t seed, uint64_t offset, uint32_t site, uint32_t row,
                               uint32_t chunk) {
  return philox(chunk + (site << 13), row, uint32_t(offset), uint32_t(offset >> 32), uint32_t(seed),
                uint32_t(seed >> 32));
}

}  // namespace abft
