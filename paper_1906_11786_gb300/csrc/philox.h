// Counter-based random bits for dropout: Philox4x32 with 7 rounds (Salmon, Moraes, Dror and Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", SC 2011; their Table 2 finds 7 rounds to pass
// BigCrush, 10 only add margin).  The bits of an element depend on (seed, call, element index)
// alone, so a backward pass draws the forward's mask again instead of reading it.
//
// One block of 4 x 32 bits serves 8 consecutive elements, 16 bits each: at 32 bits an element the
// integer multiplies of the generator, and no longer HBM, would bound a bf16 pass.  A drop
// probability is therefore a multiple of 2^-16, and the kept elements are scaled by the inverse of
// the probability that is really applied.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace bg {

// A dropout as the kernels take it: element i is kept iff its 16 bits are >= thr.
struct Drop {
  uint32_t k0, k1;  // key: the seed
  uint32_t c2, c3;  // upper half of the counter: the call
  uint32_t thr;     // round(p 2^16), 0 = everything kept, 65536 = nothing
  uint32_t lim;     // thr 2^16 - 1: 16 bits in the upper half of a word are kept iff the word is larger
  float scale;      // 65536 / (65536 - thr), 0 when nothing is kept
};

inline Drop make_drop(float p, int64_t seed, int64_t call) {
  Drop d;
  d.k0 = (uint32_t)seed;
  d.k1 = (uint32_t)((uint64_t)seed >> 32);
  d.c2 = (uint32_t)call;
  d.c3 = (uint32_t)((uint64_t)call >> 32);
  d.thr = (uint32_t)((double)p * 65536.0 + 0.5);
  d.lim = (d.thr << 16) - 1u;
  d.scale = d.thr < 65536u ? (float)(65536.0 / (65536.0 - d.thr)) : 0.f;
  return d;
}

// The 128 bits of elements 8 b .. 8 b + 7: element 8 b + j has bits 16 (j % 2) .. of word j / 2.
__device__ __forceinline__ uint4 philox_block(const Drop& d, uint64_t b) {
  uint32_t c0 = (uint32_t)b, c1 = (uint32_t)(b >> 32), c2 = d.c2, c3 = d.c3;
  uint32_t k0 = d.k0, k1 = d.k1;
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t m0 = (uint64_t)0xD2511F53u * c0, m1 = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(m1 >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)m1;
    c2 = (uint32_t)(m0 >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)m0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

// v[j] <- v[j] * scale where element 8 b + j is kept, 0 where it is dropped (also where v[j] is not
// finite).
__device__ __forceinline__ void drop8(const Drop& d, uint64_t b, float scale, float* v) {
  const uint4 w = philox_block(d, b);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = (u[j] << 16) > d.lim ? v[2 * j] * scale : 0.f;
    v[2 * j + 1] = u[j] > d.lim ? v[2 * j + 1] * scale : 0.f;
  }
}

}  // namespace bg
