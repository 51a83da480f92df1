// The counter-based generator behind dropout: Philox4x32-10 (J. Salmon, M.
// Moraes, R. Dror, D. Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// SC 2011).  A mask is a function of (seed, step, site, element) alone, so a
// checkpointed step's re-run and backward form the first forward's mask again
// and nothing stores it.
//
// Element e takes the 16-bit half e % 8 of block e / 8 (eight elements a
// block; half h = bits 16 (h % 2) .. of word h / 2) and is kept when the half
// is at least the threshold T = round(65536 p).  Sixteen bits an element: ten
// rounds are 20 32x32 -> 64-bit products, which at four elements a block would
// outweigh the memory traffic of a bf16 tensor; p is met to 2^-17, and the
// scale 65536 / (65536 - T) of the kept ones goes by T, so the mean is exact.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ckpt {

// Dropout as a kernel takes it: thr = (T << 16) - 1; rng (device: seed, step)
// null for none (T = 0).  T = 65536 keeps nothing: thr = 2^32 - 1.
struct DropArgs {
  const uint64_t *rng;
  uint32_t site, thr;
  float scale;
};

struct DropKey {
  uint32_t k0, k1, s0, s1;  // seed, step
};

__device__ __forceinline__ DropKey drop_key(const DropArgs &d) {
  DropKey k{0, 0, 0, 0};
  if (d.rng) {
    const uint64_t seed = d.rng[0], step = d.rng[1];
    k = DropKey{uint32_t(seed), uint32_t(seed >> 32), uint32_t(step), uint32_t(step >> 32)};
  }
  return k;
}

__device__ __forceinline__ void philox(const DropKey &k, uint32_t blk, uint32_t site, uint32_t w[4]) {
  uint32_t c0 = blk, c1 = site, c2 = k.s0, c3 = k.s1, k0 = k.k0, k1 = k.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = uint64_t(c0) * 0xD2511F53u, b = uint64_t(c2) * 0xCD9E8D57u;
    c0 = __builtin_amdgcn_bitop3_b32(uint32_t(b >> 32), c1, k0, 0x96);  // the three's exclusive or
    c1 = uint32_t(b);
    c2 = __builtin_amdgcn_bitop3_b32(uint32_t(a >> 32), c3, k1, 0x96);
    c3 = uint32_t(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  w[0] = c0;
  w[1] = c1;
  w[2] = c2;
  w[3] = c3;
}

// v[0..8) of one block: kept and scaled, or zero (whatever the dropped value)
__device__ __forceinline__ void drop8(const DropArgs &d, const DropKey &k, uint32_t blk, float v[8]) {
  uint32_t w[4];
  philox(k, blk, d.site, w);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    v[2 * q] = (w[q] << 16) > d.thr ? v[2 * q] * d.scale : 0.f;
    v[2 * q + 1] = w[q] > d.thr ? v[2 * q + 1] * d.scale : 0.f;
  }
}

// the same for the single element e (below 2^35)
__device__ __forceinline__ float drop1(const DropArgs &d, const DropKey &k, uint64_t e, float v) {
  uint32_t w[4];
  philox(k, uint32_t(e >> 3), d.site, w);
  const int h = int(e & 7);
  const uint32_t word = h < 4 ? (h < 2 ? w[0] : w[1]) : (h < 6 ? w[2] : w[3]);
  return ((h & 1) ? word : word << 16) > d.thr ? v * d.scale : 0.f;
}

}  // namespace ckpt
