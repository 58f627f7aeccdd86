// 16-byte vectors of the storage types: VEC elements loaded, stored and
// converted at once (VEC = 1: one element, for what is not aligned).
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

template <typename TS, int VEC>
struct vec;

template <typename TS>
struct vec<TS, 1> {
    __device__ __forceinline__ static void load(const TS *p, float *f) { f[0] = st<TS>::load(p, 0); }
    __device__ __forceinline__ static void store(TS *p, const float *f) { st<TS>::store(p, 0, f[0]); }
};

template <>
struct vec<float, 4> {
    __device__ __forceinline__ static void load(const float *p, float *f) {
        const f32x4 v = *(const f32x4 *)p;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            f[k] = v[k];
    }
    __device__ __forceinline__ static void store(float *p, const float *f) {
        *(f32x4 *)p = f32x4{f[0], f[1], f[2], f[3]};
    }
};

template <>
struct vec<bf16_t, 8> {
    __device__ __forceinline__ static void load(const bf16_t *p, float *f) {
        const uint4 v = *(const uint4 *)p;
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f[2 * k] = __uint_as_float(w[k] << 16);
            f[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ static void store(bf16_t *p, const float *f) {
        *(uint4 *)p = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]),
                                 pack_bf16(f[6], f[7]));
    }
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes that go past the caches' usual order of eviction, for a tensor too
// large for whoever reads it next to find it there.
__device__ __forceinline__ void stream(float *p, const float *f) {
    __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, (f32x4 *)p);
}
__device__ __forceinline__ void stream(bf16_t *p, const float *f) {
    __builtin_nontemporal_store(u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]),
                                      pack_bf16(f[6], f[7])},
                                (u32x4 *)p);
}
__device__ __forceinline__ void load_past(const float *p, float *f) {
    const f32x4 v = __builtin_nontemporal_load((const f32x4 *)p);
#pragma unroll
    for (int k = 0; k < 4; ++k)
        f[k] = v[k];
}
__device__ __forceinline__ void load_past(const bf16_t *p, float *f) {
    const u32x4 v = __builtin_nontemporal_load((const u32x4 *)p);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        f[2 * k] = __uint_as_float(v[k] << 16);
        f[2 * k + 1] = __uint_as_float(v[k] & 0xffff0000u);
    }
}

template <typename TS>
__device__ __forceinline__ void store16(TS *p, const float *f, bool past) {
    if (past)
        stream(p, f);
    else
        vec<TS, vec_of<TS>()>::store(p, f);
}

// Outputs from this size on are streamed: no L2 (4 MB for each of eight XCDs)
// keeps them for their reader, and their lines do not push out what this
// kernel reads again.
constexpr long STREAM_BYTES = 32L << 20;

} // namespace lstmss
