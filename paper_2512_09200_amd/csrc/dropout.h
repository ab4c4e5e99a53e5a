// Dropout's generator: which elements stay is a function of the seed, the
// step, the call's site and the element's place, so the backward pass makes
// the mask again and none is stored.
//
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as
// easy as 1, 2, 3", 2011): key = the seed's two words, counter = (column / 8,
// row, site, low word of the step).  The block's 128 bits are eight 16-bit
// numbers, word e / 2, low half first, for the eight neighbouring columns;
// element e stays where its number is >= t.  Sixteen bits an element instead of
// thirty-two halve the generator's work, which would otherwise be above the
// memory time of 2-byte elements (ten rounds of two 32 x 32 products); the
// probability is then a multiple of 2^-16, and the factor is that of the
// probability taken, so the mean is exact.
#pragma once
#include "common.h"

namespace lat {

struct DropArgs {
  uint32_t t = 0;                     // of 65536; 0: nothing is dropped
  float factor = 1.f;                 // 65536 / (65536 - t)
  uint32_t site = 0;
  const uint64_t* rng = nullptr;      // device: seed, step
};

struct DropKey { uint32_t k0, k1, site, step; };
__device__ inline DropKey drop_key(const DropArgs& d) {
  if (d.t == 0) return {0u, 0u, 0u, 0u};
  const uint64_t seed = d.rng[0], step = d.rng[1];
  // uniform over the launch: into scalar registers, the key's additions with them
  return {(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)seed),
          (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(seed >> 32)), d.site,
          (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)step)};
}

__device__ inline void philox(const DropKey& key, uint32_t group, uint32_t row, uint32_t (&w)[4]) {
  uint32_t c0 = group, c1 = row, c2 = key.site, c3 = key.step, k0 = key.k0, k1 = key.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)b;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  w[0] = c0; w[1] = c1; w[2] = c2; w[3] = c3;
}

// x[e] * factor where it stays, 0 elsewhere (whatever x[e] is)
__device__ inline void drop8(const DropArgs& d, const DropKey& key, uint32_t group, uint32_t row, float (&x)[8]) {
  uint32_t w[4];
  philox(key, group, row, w);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t n = e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
    const float y = x[e] * d.factor;
    x[e] = n >= d.t ? y : 0.f;
  }
}

}  // namespace lat
