// The counter-based generator of dropout: which elements of a tensor are dropped is computed
// where it is needed and never stored, so a backward pass draws the mask of its forward.
//
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// SC 2011): ten rounds of two 32 x 32 -> 64-bit products turn a 128-bit counter and a 64-bit
// key into 128 random bits.  Element e takes counter (e / 8, offset), each 64 bits, low words
// first, under the key `seed`; the 128 bits are eight 16-bit draws, low halves first, and
// element e takes draw e % 8.  16 bits a draw, so that one block serves the 16 bytes of eight
// bf16 elements: p is the nearest multiple of 2^-16 (off by at most 2^-17), and the scale of
// what is kept, 65536 / (65536 - thr), is that of the p in use, so expectations stay.
#pragma once

#include "ec_common.h"
#include "ec_kernels.h"

namespace ec {

// The draws of elements 8 block .. 8 block + 7 (two to a word, low half first).
__device__ __forceinline__ u32x4 dropout_block(uint64_t block, uint64_t seed, uint64_t offset) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32);
  uint32_t c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

// v[u] = kept ? v[u] * scale : 0 for the eight elements of a block.  A dropped element is
// zero whatever it holds (infinities and NaN too): selected, not multiplied.
__device__ __forceinline__ void dropout_apply(float v[8], u32x4 w, uint32_t thr, float scale) {
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const uint32_t draw = (u & 1) ? w[u >> 1] >> 16 : w[u >> 1] & 0xffffu;
    v[u] = draw >= thr ? v[u] * scale : 0.f;
  }
}

}  // namespace ec
