// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as
// easy as 1, 2, 3", 2011) and the dropout mask made of it.
#pragma once

#include "common.h"
#include "language.h"

namespace lstmss {

// One instruction on gfx950 (truth table of a ^ b ^ c).
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
    return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
}

// The 128 bits of one counter: ten rounds of two 32 x 32 -> 64 products.
__device__ __forceinline__ void philox(uint64_t counter, uint32_t k0, uint32_t k1, uint32_t out[4]) {
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = 0, c3 = 0;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = xor3((uint32_t)(b >> 32), c1, k0);
        c1 = (uint32_t)b;
        c2 = xor3((uint32_t)(a >> 32), c3, k1);
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0;
    out[1] = c1;
    out[2] = c2;
    out[3] = c3;
}

// Dropout of the VEC elements e .. e + VEC - 1 (16 bytes of a type: VEC is 4
// or 8, e a multiple of it) of a mask that repeats, if at all, after a
// multiple of 8: +0 where dropped, whatever f holds.  Eight elements share a
// counter.  Both halves of a word are compared in its high half.
template <int VEC>
__device__ __forceinline__ void drop_whole(const DropArgs &d, long e, float *f) {
    uint32_t w[4];
    const long m = d.period > 0 ? e % d.period : e;
    philox(d.counter + (uint64_t)(m >> 3), d.key0, d.key1, w);
    if (VEC == 4 && (m & 4)) {
        w[0] = w[2];
        w[1] = w[3];
    }
    const uint32_t thr = d.thr << 16;
#pragma unroll
    for (int k = 0; k < VEC; ++k)
        f[k] = (k & 1 ? w[k >> 1] : w[k >> 1] << 16) >= thr ? f[k] * d.scale : 0.f;
}

// The same for any mask.  One that repeats after no multiple of 8 takes a
// generator and a 64-bit remainder for each element: four times the time of a
// dropout over bf16, twice that of one over fp32.
template <int VEC>
__device__ __forceinline__ void drop_any(const DropArgs &d, long e, float *f) {
    if (d.thr == 0)
        return;
    if ((d.period & 7) == 0)
        return drop_whole<VEC>(d, e, f);
    uint32_t w[4];
#pragma unroll 1
    for (int k = 0; k < VEC; ++k) {
        const long m = (e + k) % d.period;
        philox(d.counter + (uint64_t)(m >> 3), d.key0, d.key1, w);
        const int h = (int)(m & 7);
        const uint32_t word = h < 4 ? (h < 2 ? w[0] : w[1]) : (h < 6 ? w[2] : w[3]);
        f[k] = (h & 1 ? word >> 16 : word & 0xffffu) >= d.thr ? f[k] * d.scale : 0.f;
    }
}

} // namespace lstmss
