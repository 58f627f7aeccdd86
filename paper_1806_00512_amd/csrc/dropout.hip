// Dropout whose mask is a function of the element's index.
#include <algorithm>

#include "common.h"
#include "language.h"
#include "philox.h"
#include "vec.h"

namespace lstmss {

namespace {

// 16 bytes of elements to a thread at a time.  WHOLE: both tensors lie on
// 16-byte boundaries and the mask repeats after a multiple of 8 if at all.
template <typename TS, bool WHOLE>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs d, long n, const TS *x, TS *y, bool past) {
    constexpr int VEC = vec_of<TS>();
    const long groups = (n + VEC - 1) / VEC;
    for (long q = blockIdx.x * 256L + threadIdx.x; q < groups; q += (long)gridDim.x * 256) {
        const long e = q * VEC;
        float f[VEC];
        if (WHOLE && e + VEC <= n) {
            vec<TS, VEC>::load(x + e, f);
            drop_whole<VEC>(d, e, f);
            store16(y + e, f, past);
        } else {
            for (int k = 0; k < VEC; ++k)
                f[k] = e + k < n ? st<TS>::load(x, e + k) : 0.f;
            drop_any<VEC>(d, e, f);
            for (int k = 0; k < VEC; ++k)
                if (e + k < n)
                    st<TS>::store(y, e + k, f[k]);
        }
    }
}

template <typename TS>
hipError_t run(const DropArgs &d, long n, const TS *x, TS *y, hipStream_t s) {
    const dim3 grid((unsigned)std::min(ceil_div(n, 256L * vec_of<TS>()), 8192L)), blk(256);
    const bool past = n * st<TS>::bytes >= STREAM_BYTES;
    if ((uintptr_t)x % 16 == 0 && (uintptr_t)y % 16 == 0 && d.period % 8 == 0)
        hipLaunchKernelGGL((dropout_kernel<TS, true>), grid, blk, 0, s, d, n, x, y, past);
    else
        hipLaunchKernelGGL((dropout_kernel<TS, false>), grid, blk, 0, s, d, n, x, y, past);
    return hipGetLastError();
}

} // namespace

hipError_t launch_dropout(const DropArgs &d, long n, const void *x, void *y, bool bf16,
                          hipStream_t s) {
    return bf16 ? run(d, n, (const bf16_t *)x, (bf16_t *)y, s) : run(d, n, (const float *)x, (float *)y, s);
}

} // namespace lstmss
