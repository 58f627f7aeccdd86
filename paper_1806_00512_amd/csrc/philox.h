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

// f[k] scaled where the 16 bits number k of a counter's 128 reach the
// threshold, else +0.  (Both halves of a word are compared in its high half.)
__device__ __forceinline__ void drop_apply(const DropArgs &d, const uint32_t w[4], float *f) {
    const uint32_t thr = d.thr << 16;
#pragma unroll
    for (int k = 0; k < 8; ++k)
        f[k] = (k & 1 ? w[k >> 1] : w[k >> 1] << 16) >= thr ? f[k] * d.scale : 0.f;
}

// The same for masks that repeat, if at all, after a multiple of 8.
__device__ __forceinline__ void drop8_whole(const DropArgs &d, long e, float *f) {
    uint32_t w[4];
    const long m = d.period > 0 ? e % d.period : e;
    philox(d.counter + (uint64_t)(m >> 3), d.key0, d.key1, w);
    drop_apply(d, w, f);
}

// Dropout of the eight elements e .. e + 7 (e a multiple of 8): +0 where
// dropped, whatever f holds.  One counter gives all eight, unless the mask
// repeats after a length that is no multiple of 8.
__device__ __forceinline__ void drop8(const DropArgs &d, long e, float *f) {
    if (d.thr == 0)
        return;
    if ((d.period & 7) == 0)
        return drop8_whole(d, e, f);
    uint32_t w[4];
#pragma unroll 1
    for (int k = 0; k < 8; ++k) {
        const long m = (e + k) % d.period;
        philox(d.counter + (uint64_t)(m >> 3), d.key0, d.key1, w);
        const int h = (int)(m & 7);
        const uint32_t word = h < 4 ? (h < 2 ? w[0] : w[1]) : (h < 6 ? w[2] : w[3]);
        f[k] = (h & 1 ? word >> 16 : word & 0xffffu) >= d.thr ? f[k] * d.scale : 0.f;
    }
}

} // namespace lstmss
