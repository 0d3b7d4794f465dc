// Dropout masks from a counter-based generator (Philox4x32 of ten rounds; Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as
// easy as 1, 2, 3", 2011), so that no mask is stored: forward and backward form it from the position alone.  One generator call, of counter
// (column / 8, row, site, step) under the key `seed`, gives 128 bits, sixteen for each of eight neighbouring columns; an element is kept where its
// number is at least `threshold` = the probability times 2^16, rounded.  With 32 bits an element the generator's twenty 32 x 32 bit products, quarter
// rate each, would take longer than the memory that the element moves.
#pragma once
#include "dp_device.h"

namespace dp {

struct DropK {
  const uint64_t* rng;      // [device] {seed, step}; read by the kernel, so that a captured graph sees what a replay finds there
  uint32_t threshold;       // of 65536; 0: nothing is dropped and rng is not read
  uint32_t site, row0;
  float up;                 // 65536 / (65536 - threshold); 0 if everything is dropped
};

struct DropKey { uint32_t k0, k1, step; };
__device__ __forceinline__ DropKey drop_key(const DropK& d) {
  if (d.threshold == 0) return {0, 0, 0};
  const uint64_t seed = d.rng[0];
  return {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)d.rng[1]};
}

// The sixteen bits of columns 8 group .. + 7 of a row: column 8 group + j has bits 16 (j & 1) .. of word j / 2.
__device__ __forceinline__ u32x4 drop_bits(const DropKey& key, uint32_t group, uint32_t row, uint32_t site) {
  uint32_t c0 = group, c1 = row, c2 = site, c3 = key.step, k0 = key.k0, k1 = key.k1;
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
  return u32x4{c0, c1, c2, c3};
}

// v[j] = kept ? v[j] * up : 0.  A dropped element contributes zero whatever it holds.
__device__ __forceinline__ void drop8(const DropK& d, const DropKey& key, uint32_t group, uint32_t row, float (&v)[8]) {
  if (d.threshold == 0) return;
  const u32x4 w = drop_bits(key, group, d.row0 + row, d.site);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t u = j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xFFFFu;
    v[j] = u >= d.threshold ? v[j] * d.up : 0.f;
  }
}

}  // namespace dp
