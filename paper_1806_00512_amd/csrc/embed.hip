// Embedding lookup into the batch-last layout, and its gradient by sorted tokens.
#include <algorithm>

#include "common.h"
#include "language.h"
#include "philox.h"

namespace lstmss {

namespace {

// x[t][i][b] = scale * E[tokens[t][b]][i]: one thread for each element.
template <typename TS>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a) {
    const long n = (long)a.T * a.I * a.B;
    const TS *E = (const TS *)a.E;
    for (long e = blockIdx.x * 256L + threadIdx.x; e < n; e += (long)gridDim.x * 256) {
        const long ti = e / a.B;
        const int b = (int)(e - ti * a.B);
        const int t = (int)(ti / a.I), i = (int)(ti - (long)t * a.I);
        const int32_t v = a.tokens[(long)t * a.B + b];
        const float f = (uint32_t)v < (uint32_t)a.V ? st<TS>::load(E, (long)v * a.I + i) * a.scale : 0.f;
        st<TS>::store((TS *)a.x, e, drop_one(a.drop, e, f));
    }
}

// order[r] = the position whose (token, position) has rank r: each position
// counts those before it.  Tokens outside [0, V) come last, as V.
__global__ __launch_bounds__(256) void rank_kernel(const int32_t *tokens, int N, int V, int32_t *key,
                                                   int32_t *order) {
    const int p = blockIdx.x * 256 + threadIdx.x;
    if (p >= N)
        return;
    const uint32_t mine = min((uint32_t)tokens[p], (uint32_t)V);
    int r = 0;
    for (int q = 0; q < N; ++q) {
        const uint32_t other = min((uint32_t)tokens[q], (uint32_t)V);
        r += other < mine || (other == mine && q < p);
    }
    key[r] = (int32_t)mine;
    order[r] = p;
}

// First r with key[r] >= v.
__device__ __forceinline__ int lower_bound(const int32_t *key, int N, int v) {
    int lo = 0, hi = N;
    while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (key[mid] < v)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}

// dE[v][i]: one work-group for each row, summing its positions in order.
__global__ __launch_bounds__(256) void embed_grad_kernel(EmbedGradArgs a, int N, const int32_t *key,
                                                         const int32_t *order) {
    const int v = blockIdx.x;
    const int r0 = lower_bound(key, N, v), r1 = lower_bound(key, N, v + 1);
    if (a.accumulate && r0 == r1)
        return;
    for (int i = threadIdx.x; i < a.I; i += 256) {
        float sum = 0.f;
        for (int r = r0; r < r1; ++r) {
            const int t = order[r] / a.B, b = order[r] - t * a.B;
            const long e = ((long)t * a.I + i) * a.B + b;
            sum += drop_one(a.drop, e, a.dX[e]);
        }
        float *p = a.dE + (long)v * a.I + i;
        *p = a.accumulate ? *p + sum * a.scale : sum * a.scale;
    }
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

} // namespace

hipError_t launch_embed(const EmbedArgs &a, bool bf16, hipStream_t s) {
    const long n = (long)a.T * a.I * a.B;
    const dim3 grid((unsigned)std::min(ceil_div(n, 256L), 8192L));
    if (bf16)
        hipLaunchKernelGGL(embed_kernel<bf16_t>, grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL(embed_kernel<float>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

size_t embed_grad_ws(int T, int B, int I, int V) {
    (void)I;
    (void)V;
    return 2 * align256((size_t)T * B * 4);
}

hipError_t launch_embed_grad(const EmbedGradArgs &a, hipStream_t s) {
    const int N = a.T * a.B;
    int32_t *key = (int32_t *)a.ws;
    int32_t *order = (int32_t *)((char *)a.ws + align256((size_t)N * 4));
    hipLaunchKernelGGL(rank_kernel, dim3((unsigned)ceil_div(N, 256)), dim3(256), 0, s, a.tokens, N, a.V, key, order);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(embed_grad_kernel, dim3((unsigned)a.V), dim3(256), 0, s, a, N, key, order);
    return hipGetLastError();
}

} // namespace lstmss
