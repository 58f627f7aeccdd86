// Losses on batch-last logits [T][V][B]: log softmax over the middle axis at
// the targets, per-token terms, gradient in the logits.
//
//   m = max_v x_v,  s = sum_v exp(x_v - m),  logp = x_y - m - log s
//   dL/dx_v = dlogp * ([v = y] - exp(x_v - m) / s)
#include <algorithm>

#include "common.h"
#include "language.h"

namespace lstmss {

namespace {

// Running maximum and sum of exponentials of a column.
struct Stat {
    float m, s;
};

__device__ __forceinline__ Stat stat_empty() { return {-INFINITY, 0.f}; }

// exp(x - m) with the maximum -inf of a column that holds nothing else read as 0.
__device__ __forceinline__ float exp_from(float x, float m) {
    return __expf(x - (m == -INFINITY ? 0.f : m));
}

__device__ __forceinline__ Stat stat_join(Stat a, Stat b) {
    const float m = fmaxf(a.m, b.m);
    return {m, a.s * exp_from(a.m, m) + b.s * exp_from(b.m, m)};
}

// stat[t][b]: 64 columns to a work-group, four rows at a time.
template <typename TS>
__global__ __launch_bounds__(256) void stat_kernel(LossArgs a, Stat *stat) {
    __shared__ Stat part[4][64];
    const int groups = (a.B + 63) / 64;
    const int t = blockIdx.x / groups, b = (blockIdx.x % groups) * 64 + (threadIdx.x & 63);
    const int lane = threadIdx.x & 63, row = threadIdx.x >> 6;
    const TS *x = (const TS *)a.logits + (long)t * a.V * a.B;
    Stat q = stat_empty();
    if (b < a.B)
        for (int v = row; v < a.V; v += 4)
            q = stat_join(q, {st<TS>::load(x, (long)v * a.B + b), 1.f});
    part[row][lane] = q;
    __syncthreads();
    if (row == 0 && b < a.B) {
        for (int r = 1; r < 4; ++r)
            q = stat_join(q, part[r][lane]);
        stat[(long)t * a.B + b] = q;
    }
}

// Per token: logp, the loss term, and what the gradient kernel multiplies by:
// coef[n] = {m, dlogp / s, dlogp}; part[block] = the block's loss, in order.
struct Coef {
    float m, p, g;
};

__global__ __launch_bounds__(256) void token_kernel(LossArgs a, const Stat *stat, Coef *coef, double *part) {
    __shared__ double red[256];
    const long N = (long)a.T * a.B, n = blockIdx.x * 256L + threadIdx.x;
    double term = 0.0;
    if (n < N) {
        const Stat q = stat[n];
        const int y = a.targets[n];
        const double w = a.weights ? (double)a.weights[n] : 1.0;
        double lp = 0.0, g = 0.0;
        if ((uint32_t)y < (uint32_t)a.V && w != 0.0) {
            const int t = (int)(n / a.B);
            const long at = ((long)t * a.V + y) * a.B + (n - (long)t * a.B);
            const float x = a.bf16 ? st<bf16_t>::load((const bf16_t *)a.logits, at) : ((const float *)a.logits)[at];
            lp = ((double)x - (double)q.m) - log((double)q.s);
            if (a.mode == LOSS_XENT) {
                term = -lp;
                g = -1.0;
            } else if (a.mode == LOSS_POLICY) {
                const double A = a.adv[n];
                const double r = a.old_logp ? exp(lp - (double)a.old_logp[n]) : 1.0;
                const double c = fmin(fmax(r, 1.0 - (double)a.clip_low), 1.0 + (double)a.clip_high);
                const double gain = r * A, held = c * A;
                term = -(gain <= held || gain != gain ? gain : held);
                g = gain <= held || gain != gain ? -gain : 0.0;
                if (a.ref_logp) {
                    const double d = (double)a.ref_logp[n] - lp, e = expm1(d);
                    term += (double)a.kl * (e - d);
                    g -= (double)a.kl * e;
                }
            }
            term *= w * (double)a.scale;
            g *= w * (double)a.scale;
        }
        if (a.logp)
            a.logp[n] = (float)lp;
        coef[n] = {q.m, (float)(g / (double)q.s), (float)g};
    }
    red[threadIdx.x] = term;
    __syncthreads();
    for (int w = 128; w >= 1; w >>= 1) {
        if ((int)threadIdx.x < w)
            red[threadIdx.x] += red[threadIdx.x + w];
        __syncthreads();
    }
    if (threadIdx.x == 0)
        part[blockIdx.x] = red[0];
}

__global__ __launch_bounds__(256) void loss_sum_kernel(const double *part, int n, float *loss) {
    __shared__ double red[256];
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += 256)
        sum += part[i];
    red[threadIdx.x] = sum;
    __syncthreads();
    for (int w = 128; w >= 1; w >>= 1) {
        if ((int)threadIdx.x < w)
            red[threadIdx.x] += red[threadIdx.x + w];
        __syncthreads();
    }
    if (threadIdx.x == 0)
        *loss = (float)red[0];
}

template <typename TS>
__global__ __launch_bounds__(256) void grad_kernel(LossArgs a, const Coef *coef) {
    const long n = (long)a.T * a.V * a.B;
    const TS *x = (const TS *)a.logits;
    TS *y = (TS *)a.dlogits;
    for (long e = blockIdx.x * 256L + threadIdx.x; e < n; e += (long)gridDim.x * 256) {
        const long tv = e / a.B;
        const int b = (int)(e - tv * a.B), t = (int)(tv / a.V), v = (int)(tv - (long)t * a.V);
        const long k = (long)t * a.B + b;
        const Coef c = coef[k];
        float d = 0.f;
        if (c.g != 0.f) {
            d = -c.p * exp_from(st<TS>::load(x, e), c.m);
            if (a.targets[k] == v)
                d += c.g;
        }
        st<TS>::store(y, e, d);
    }
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

struct LossWs {
    Stat *stat;
    Coef *coef;
    double *part;
    size_t bytes;
    int parts;
};

LossWs layout(void *ws, int T, int B) {
    const size_t N = (size_t)T * B;
    char *p = (char *)ws;
    LossWs w;
    w.parts = (int)((N + 255) / 256);
    size_t at = 0;
    w.stat = (Stat *)(p + at);
    at += align256(N * sizeof(Stat));
    w.coef = (Coef *)(p + at);
    at += align256(N * sizeof(Coef));
    w.part = (double *)(p + at);
    at += align256((size_t)w.parts * 8);
    w.bytes = at;
    return w;
}

} // namespace

size_t loss_ws(int T, int B, int V, bool bf16) {
    (void)V;
    (void)bf16;
    return layout(nullptr, T, B).bytes;
}

hipError_t launch_loss(const LossArgs &a, hipStream_t s) {
    const LossWs w = layout(a.ws, a.T, a.B);
    hipError_t e;
    const dim3 blk(256), gs((unsigned)((long)a.T * ceil_div(a.B, 64)));
    if (a.bf16)
        hipLaunchKernelGGL(stat_kernel<bf16_t>, gs, blk, 0, s, a, w.stat);
    else
        hipLaunchKernelGGL(stat_kernel<float>, gs, blk, 0, s, a, w.stat);
    if ((e = hipGetLastError()) != hipSuccess)
        return e;
    hipLaunchKernelGGL(token_kernel, dim3((unsigned)w.parts), blk, 0, s, a, w.stat, w.coef, w.part);
    if ((e = hipGetLastError()) != hipSuccess)
        return e;
    if (a.loss) {
        hipLaunchKernelGGL(loss_sum_kernel, dim3(1), blk, 0, s, w.part, w.parts, a.loss);
        if ((e = hipGetLastError()) != hipSuccess)
            return e;
    }
    if (!a.dlogits)
        return hipSuccess;
    const dim3 gg((unsigned)std::min(ceil_div((long)a.T * a.V * a.B, 256L), 16384L));
    if (a.bf16)
        hipLaunchKernelGGL(grad_kernel<bf16_t>, gg, blk, 0, s, a, w.coef);
    else
        hipLaunchKernelGGL(grad_kernel<float>, gg, blk, 0, s, a, w.coef);
    return hipGetLastError();
}

} // namespace lstmss
