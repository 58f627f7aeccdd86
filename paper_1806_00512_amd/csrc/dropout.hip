// Dropout whose mask is a function of the element's index.
#include <algorithm>

#include "common.h"
#include "language.h"
#include "philox.h"

namespace lstmss {

namespace {

template <typename TS>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs d, long n, const TS *x, TS *y) {
    for (long e = blockIdx.x * 256L + threadIdx.x; e < n; e += (long)gridDim.x * 256)
        st<TS>::store(y, e, drop_one(d, e, st<TS>::load(x, e)));
}

} // namespace

hipError_t launch_dropout(const DropArgs &d, long n, const void *x, void *y, bool bf16,
                          hipStream_t s) {
    const dim3 grid((unsigned)std::min(ceil_div(n, 256L), 8192L));
    if (bf16)
        hipLaunchKernelGGL(dropout_kernel<bf16_t>, grid, dim3(256), 0, s, d, n, (const bf16_t *)x, (bf16_t *)y);
    else
        hipLaunchKernelGGL(dropout_kernel<float>, grid, dim3(256), 0, s, d, n, (const float *)x, (float *)y);
    return hipGetLastError();
}

} // namespace lstmss
