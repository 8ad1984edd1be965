// Counter-based random bits for dropout: Philox-4x32 with 7 rounds (J. Salmon et
// al., "Parallel random numbers: as easy as 1, 2, 3", SC 2011; 7 is the least
// number of rounds that the paper found to pass its statistical tests).
//
// One call turns a 128-bit counter and a 64-bit key into 128 bits: eight 16-bit
// numbers, one for each element of a group.  The counter is (group, offset) and
// the key is the seed, so a mask is a function of three numbers and is never
// stored; the backward evaluates it again.  16 bits an element instead of 32
// halve the cost of the generator, which is bound by its 32-bit products (a
// quarter of the rate of other vector operations); the drop probability is then
// a multiple of 2^-16.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace petra {

struct Rng {
  uint32_t key0, key1, off0, off1;
};

// rng: device {seed, offset}.
__device__ __forceinline__ Rng load_rng(const uint64_t* rng) {
  const uint64_t seed = rng[0], off = rng[1];
  return {static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32),
          static_cast<uint32_t>(off), static_cast<uint32_t>(off >> 32)};
}

// The 128 bits of `group`; element e of it has bits 16 e .. 16 e + 15.
__device__ __forceinline__ void philox(const Rng& r, uint64_t group, uint32_t w[4]) {
  uint32_t c0 = static_cast<uint32_t>(group), c1 = static_cast<uint32_t>(group >> 32);
  uint32_t c2 = r.off0, c3 = r.off1, k0 = r.key0, k1 = r.key1;
#pragma unroll
  for (int i = 0; i < 7; ++i) {
    const uint64_t a = static_cast<uint64_t>(c0) * 0xD2511F53u;
    const uint64_t b = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
    c0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0;
    c1 = static_cast<uint32_t>(b);
    c2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
    c3 = static_cast<uint32_t>(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  w[0] = c0; w[1] = c1; w[2] = c2; w[3] = c3;
}

// Whether element e (0 .. 7) of the group with bits w is kept: its 16 bits are at
// least `cut` = round(65536 p).  The high half is compared in place, its low bits
// under the cut's.
__device__ __forceinline__ bool kept(const uint32_t w[4], int e, uint32_t cut) {
  return (e & 1) ? w[e >> 1] >= (cut << 16) : (w[e >> 1] & 0xffffu) >= cut;
}

}  // namespace petra
