// Uniform numbers of the stochastic rounding.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ecasq {

// Philox4x32-10 (Salmon et al., SC'11) at counter c: ten rounds of
// two 32x32->64 products mixed with the other words and the round key; the key
// advances by the two Weyl increments between rounds.  (With an inlined call the
// products of the words that are zero or the same in every thread fold away:
// 18 of 20 remain for c2 = 0.)
__device__ __forceinline__ void philox4x32_10(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int rnd = 0; rnd < 10; rnd++) {
        if (rnd) {
            k0 += 0x9E3779B9u;
            k1 += 0xBB67AE85u;
        }
        // each 32 x 32 -> 64 product in one instruction (hi and lo halves)
        const uint64_t p0 = (uint64_t)0xD2511F53u * c[0];
        const uint64_t p1 = (uint64_t)0xCD9E8D57u * c[2];
        const uint32_t hi0 = (uint32_t)(p0 >> 32), lo0 = (uint32_t)p0;
        const uint32_t hi1 = (uint32_t)(p1 >> 32), lo1 = (uint32_t)p1;
        // (truth table of a three-way exclusive or, one instruction each)
        const uint32_t n0 = __builtin_amdgcn_bitop3_b32(hi1, c[1], k0, 0x96);
        const uint32_t n2 = __builtin_amdgcn_bitop3_b32(hi0, c[3], k1, 0x96);
        c[0] = n0;
        c[1] = lo1;
        c[2] = n2;
        c[3] = lo0;
    }
}

__device__ __forceinline__ double uniform53(uint32_t lo, uint32_t hi) {
    const uint64_t bits = ((((uint64_t)hi) << 32) | lo) >> 11;
    return (double)bits * 0x1p-53;
}

}  // namespace ecasq
