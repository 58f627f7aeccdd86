// Dropout whose mask is a function of the element's index: y_e = x_e / (1 - p)
// where the element's 16 bits reach p * 65536, else 0.  Bound by the memory: 105M
// elements, bf16 72 us (5.8 TB/s), fp32 149 us (5.6 TB/s), at the rate of a copy;
// Philox alone, a counter for eight elements, would take about 45 us.  A mask that
// repeats after no multiple of 8 is bound by Philox and a remainder for every
// element: 104M elements, bf16 276 us, fp32 287.
#include <algorithm>

#include "common.h"
#include "language.h"
#include "philox.h"
#include "vec.h"

namespace lstmss {

namespace {

// 16 bytes of elements to a thread at a time.  WHOLE: the mask repeats after a
// multiple of 8 if at all.  PAST: y is streamed.
template <typename TS, bool WHOLE, bool PAST>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs d, long n, const TS *x, TS *y) {
    constexpr int VEC = vec_of<TS>();
    const long groups = (n + VEC - 1) / VEC;
    for (long q = blockIdx.x * 256L + threadIdx.x; q < groups; q += (long)gridDim.x * 256) {
        const long e = q * VEC;
        const bool all = e + VEC <= n;
        float f[VEC];
        if (all)
            load16(x + e, f);
        else
            load_part(x + e, 0, (int)(n - e), f, 0.f);
        if (WHOLE)
            drop_whole<VEC>(d, e, f);
        else
            drop_any<VEC>(d, e, f);
        if (all)
            store16<PAST>(y + e, f);
        else
            store_part(y + e, 0, (int)(n - e), f);
    }
}

template <typename TS, bool PAST>
hipError_t run(const DropArgs &d, long n, const TS *x, TS *y, hipStream_t s) {
    const dim3 grid((unsigned)std::min(ceil_div(n, 256L * vec_of<TS>()), 8192L)), blk(256);
    if (d.period % 8 == 0)
        hipLaunchKernelGGL((dropout_kernel<TS, true, PAST>), grid, blk, 0, s, d, n, x, y);
    else
        hipLaunchKernelGGL((dropout_kernel<TS, false, PAST>), grid, blk, 0, s, d, n, x, y);
    return hipGetLastError();
}

template <typename TS>
hipError_t run(const DropArgs &d, long n, const void *x, void *y, hipStream_t s) {
    return n * st<TS>::bytes >= STREAM_BYTES ? run<TS, true>(d, n, (const TS *)x, (TS *)y, s)
                                             : run<TS, false>(d, n, (const TS *)x, (TS *)y, s);
}

} // namespace

hipError_t launch_dropout(const DropArgs &d, long n, const void *x, void *y, bool bf16,
                          hipStream_t s) {
    return bf16 ? run<bf16_t>(d, n, x, y, s) : run<float>(d, n, x, y, s);
}

} // namespace lstmss
