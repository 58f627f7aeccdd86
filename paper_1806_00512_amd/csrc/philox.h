// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as
// easy as 1, 2, 3", 2011) and the dropout mask made of it.
#pragma once

#include "common.h"
#include "language.h"

namespace lstmss {

// The 128 bits of one counter: ten rounds of two 32 x 32 -> 64 products.
__device__ __forceinline__ void philox(uint64_t counter, uint32_t k0, uint32_t k1, uint32_t out[4]) {
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = 0, c3 = 0;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0;
    out[1] = c1;
    out[2] = c2;
    out[3] = c3;
}

// The 16 bits number k of a counter's 128.
__device__ __forceinline__ uint32_t drop_bits(const uint32_t w[4], int k) {
    return k & 1 ? w[k >> 1] >> 16 : w[k >> 1] & 0xffffu;
}

// The element a mask index e of a drop with a period stands at.
__device__ __forceinline__ long drop_index(const DropArgs &d, long e) {
    return d.period > 0 ? e % d.period : e;
}

// Element e of a tensor, with dropout: +0 where dropped, whatever v is.
__device__ __forceinline__ float drop_one(const DropArgs &d, long e, float v) {
    if (d.thr == 0)
        return v;
    const long m = drop_index(d, e);
    uint32_t w[4];
    philox(d.counter + (uint64_t)(m >> 3), d.key0, d.key1, w);
    const int k = (int)(m & 7);
    const uint32_t word = k < 4 ? (k < 2 ? w[0] : w[1]) : (k < 6 ? w[2] : w[3]);
    const uint32_t bits = k & 1 ? word >> 16 : word & 0xffffu;
    return bits >= d.thr ? v * d.scale : 0.f;
}

} // namespace lstmss
