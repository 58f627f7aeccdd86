// 16-byte vectors of the storage types: VEC elements (4 fp32 or 8 bf16)
// loaded, converted and stored at once, from any element on: the target's
// memory instructions need no more than the element's own alignment, and cost
// the same where the 16 bytes lie in one line.
#pragma once

#include "common.h"

namespace lstmss {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <typename TS>
constexpr int vec_of() {
    return 16 / st<TS>::bytes;
}

// Two floats to bf16, nearest even (one instruction on gfx950).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_f32 __attribute__((aligned(4)));
typedef u32x4 u32x4_bf16 __attribute__((aligned(2)));

template <typename TS>
struct vec;

template <>
struct vec<float> {
    typedef u32x4_f32 raw;
    __device__ __forceinline__ static void open(u32x4 v, float *f) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            f[k] = __uint_as_float(v[k]);
    }
    __device__ __forceinline__ static u32x4 close(const float *f) {
        return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
};

template <>
struct vec<bf16_t> {
    typedef u32x4_bf16 raw;
    __device__ __forceinline__ static void open(u32x4 v, float *f) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f[2 * k] = __uint_as_float(v[k] << 16);
            f[2 * k + 1] = __uint_as_float(v[k] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ static u32x4 close(const float *f) {
        return u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
    }
};

// PAST: past the caches' usual order of eviction, for a tensor too large for
// whoever reads it next to find it there.  (A template's choice: the compiler
// makes one ordinary access of two branches that differ in this alone.)
template <bool PAST = false, typename TS>
__device__ __forceinline__ void load16(const TS *p, float *f) {
    typedef typename vec<TS>::raw raw;
    if constexpr (PAST)
        vec<TS>::open(__builtin_nontemporal_load((const raw *)p), f);
    else
        vec<TS>::open(*(const raw *)p, f);
}

template <bool PAST = false, typename TS>
__device__ __forceinline__ void store16(TS *p, const float *f) {
    typedef typename vec<TS>::raw raw;
    const raw v = vec<TS>::close(f);
    if constexpr (PAST)
        __builtin_nontemporal_store(v, (raw *)p);
    else
        *(raw *)p = v;
}

// Of VEC elements from p the ones in [from, to): the others `else_`, and not touched.
template <typename TS>
__device__ __forceinline__ void load_part(const TS *p, int from, int to, float *f, float else_) {
#pragma unroll
    for (int k = 0; k < vec_of<TS>(); ++k)
        f[k] = k >= from && k < to ? st<TS>::load(p, k) : else_;
}

template <typename TS>
__device__ __forceinline__ void store_part(TS *p, int from, int to, const float *f) {
#pragma unroll
    for (int k = 0; k < vec_of<TS>(); ++k)
        if (k >= from && k < to)
            st<TS>::store(p, k, f[k]);
}

// Outputs from this size on are streamed past the caches: no L2 (4 MB for each
// of eight XCDs) keeps them for their reader, and their lines do not push out
// what this kernel reads again.
constexpr long STREAM_BYTES = 32L << 20;

} // namespace lstmss
