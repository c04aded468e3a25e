// The counter-based generator of the dropouts: Philox4x32-10 (Salmon, Moraes, Dror and
// Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011).  A block of four 32-bit
// words is a function of a counter and a key alone, so an element's word follows from
// its place: no mask is stored, and a backward pass makes the same words again.
//
// Element i of a dropout takes 16-bit word i % 8 (the low half of a 32-bit word first)
// of the block with counter (i / 8, site, step low, step high) and key (seed low, seed
// high).  16 bits an element: a block's ten rounds are 20 products of 32 x 32 bits, and
// with 32 bits an element they would take longer than the element's bytes do.
#pragma once

#include "common.hpp"

namespace fp16k {

struct Drop {
  const uint64_t* state;  // seed and step, device memory
  uint32_t site;
  uint32_t threshold;     // words at least this large are kept; 0: no dropout
  float scale;            // of kept values, 65536 / (65536 - threshold)
};

// threshold and scale of a drop probability in [0, 1]
inline Drop make_drop(float p, uint32_t site, const uint64_t* state) {
  const uint32_t t = (uint32_t)((double)p * 65536.0 + 0.5);
  return {state, site, t, t < 65536 ? (float)(65536.0 / (double)(65536 - t)) : 0.0f};
}

struct PhiloxBlock {
  uint32_t w[4];
};

// The words of group g of 8 elements.  XOR3: a round's two differences of three words in one
// instruction each (kernels that hold many registers spill with it).
template <bool XOR3 = false>
__device__ __forceinline__ PhiloxBlock philox(uint32_t g, uint32_t site, uint64_t step,
                                              uint64_t seed) {
  uint32_t c0 = g, c1 = site, c2 = (uint32_t)step, c3 = (uint32_t)(step >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    const uint32_t bh = (uint32_t)(b >> 32), ah = (uint32_t)(a >> 32);
    c0 = XOR3 ? __builtin_amdgcn_bitop3_b32(bh, c1, k0, 0x96) : bh ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = XOR3 ? __builtin_amdgcn_bitop3_b32(ah, c3, k1, 0x96) : ah ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}

// Whether element j of a block's eight is kept.
__device__ __forceinline__ bool kept(const PhiloxBlock& b, int j, uint32_t threshold) {
  return ((b.w[j >> 1] >> (16 * (j & 1))) & 0xFFFFu) >= threshold;
}

}  // namespace fp16k
