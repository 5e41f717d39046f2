// Device helper: the random bits of dropout, from a counter instead of a state.
//
// Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", SC 2011): a round takes the two 64-bit products
// of words 0 and 2 with constants, and mixes their halves with words 1 and 3 and
// the round's key, which grows by a constant a round.  A counter (column / 8, row,
// stream low, stream high) yields 4 words, 16 bits for each of eight columns.  So
// a mask is a function of the seed and of an element's place in the whole matrix:
// the gradient, another launch shape or another part of the rows forms it anew.
// 16 bits set the share that is dropped to 1 / 65536; 32 would double the
// products, which are a quarter of the rate of other instructions: 20 of them a
// counter are half of its time.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace partir {

struct Dropout {
  const uint64_t* seed;    // device: key, stream; NULL: nothing is dropped
  uint32_t row0;           // number of the first row in the whole matrix
  uint32_t kept;           // of 65536
  float factor;            // 65536 / kept (0 for 0)
};

struct Philox {
  uint32_t k0, k1, c2, c3;
  __device__ __forceinline__ void init(const uint64_t* seed) {   // the same address in every lane: scalar registers
    const uint64_t key = seed[0], stream = seed[1];
    k0 = __builtin_amdgcn_readfirstlane((uint32_t)key);
    k1 = __builtin_amdgcn_readfirstlane((uint32_t)(key >> 32));
    c2 = __builtin_amdgcn_readfirstlane((uint32_t)stream);
    c3 = __builtin_amdgcn_readfirstlane((uint32_t)(stream >> 32));
  }
  // Which of columns 8 col8 .. 8 col8 + 7 of a row are kept: bit e for column e.
  __device__ __forceinline__ uint32_t keep8(uint32_t col8, uint32_t row, uint32_t kept) const {
    uint32_t x0 = col8, x1 = row, x2 = c2, x3 = c3, r0 = k0, r1 = k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      const uint64_t a = (uint64_t)x0 * 0xD2511F53u, b = (uint64_t)x2 * 0xCD9E8D57u;
      x0 = (uint32_t)(b >> 32) ^ x1 ^ r0;
      x1 = (uint32_t)b;
      x2 = (uint32_t)(a >> 32) ^ x3 ^ r1;
      x3 = (uint32_t)a;
      r0 += 0x9E3779B9u;
      r1 += 0xBB67AE85u;
    }
    const uint32_t x[4] = {x0, x1, x2, x3};
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      bits |= (uint32_t)((x[i] & 0xFFFFu) < kept) << (2 * i) | (uint32_t)((x[i] >> 16) < kept) << (2 * i + 1);
    return bits;
  }
};

}  // namespace partir
