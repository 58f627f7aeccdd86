// Dropout whose mask is a function of the element's index.
#include <algorithm>

#include "common.h"
#include "language.h"
#include "philox.h"
#include "vec.h"

namespace lstmss {

namespace {

template <typename TS>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs d, long n, const TS *x, TS *y, bool aligned) {
    const long groups = (n + 7) >> 3;
    for (long q = blockIdx.x * 256L + threadIdx.x; q < groups; q += (long)gridDim.x * 256) {
        const long e = q * 8;
        float f[8];
        const bool whole = aligned && e + 8 <= n;
        if (whole) {
            load8(x + e, f);
        } else {
            for (int k = 0; k < 8; ++k)
                f[k] = e + k < n ? st<TS>::load(x, e + k) : 0.f;
        }
        drop8(d, e, f);
        if (whole) {
            store8(y + e, f);
        } else {
            for (int k = 0; k < 8; ++k)
                if (e + k < n)
                    st<TS>::store(y, e + k, f[k]);
        }
    }
}

} // namespace

hipError_t launch_dropout(const DropArgs &d, long n, const void *x, void *y, bool bf16,
                          hipStream_t s) {
    const dim3 grid((unsigned)std::min(ceil_div(n, 2048L), 8192L));
    const bool aligned = (uintptr_t)x % 16 == 0 && (uintptr_t)y % 16 == 0;
    if (bf16)
        hipLaunchKernelGGL(dropout_kernel<bf16_t>, grid, dim3(256), 0, s, d, n, (const bf16_t *)x, (bf16_t *)y, aligned);
    else
        hipLaunchKernelGGL(dropout_kernel<float>, grid, dim3(256), 0, s, d, n, (const float *)x, (float *)y, aligned);
    return hipGetLastError();
}

} // namespace lstmss
