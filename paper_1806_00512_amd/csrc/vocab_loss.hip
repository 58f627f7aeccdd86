// Losses on batch-last logits [T][V][B]: log softmax over the middle axis at
// the targets, per-token terms, gradient in the logits.
//
//   m = max_v x_v,  s = sum_v exp(x_v - m),  logp = x_y - m - log s
//   dL/dx_v = dlogp * ([v = y] - exp(x_v - m) / s)
//
// Three kernels: partial (m, s) of every column over a chunk of rows; the
// per-token terms (the chunks' joined (m, s), logp, loss term, dlogp), which for
// small logits are one; the gradient, one of whose work-groups also sums the
// loss.  The gradient's
// work-groups go through the logits from the end, where the first kernel left
// off: what of them is still in the last-level cache need not come from memory
// again.  A step's logits are V * B elements in one piece, columns
// fastest, so a thread that walks a piece in strides of whole rows keeps its
// columns: their running (m, s), or their (m, -dlogp / s), stay in registers,
// whatever B is.
//
// Bound by the memory, which gives the logits twice and takes the gradient
// once.  Loss and gradient of 50 x 32000 x 128 logits (us): bf16 199 (1.23 GB, 6.2
// TB/s; sums 78, tokens 5, gradient 123), fp32 381 (6.4 TB/s; 128, 6, 252);
// 35 x 10000 x 20 fp32 22.8 (9, 4, 11).  Joining the token's
// terms to the gradient's work-groups, which saves a launch, measured slower
// (23 to 48 us against 22 to 32): fp64 logarithms and exponentials of all tokens
// then wait for one work-group.
#include <algorithm>
#include <cfloat>
#include <numeric>
#include <type_traits>

#include "common.h"
#include "language.h"
#include "vec.h"

namespace lstmss {

namespace {

constexpr int NT = 256; // threads of a work-group at most

// Reference and sum of exponentials of a column: sum exp(x - m), where m is a
// value seen or up to GROW below the largest one.  Empty: the lowest finite
// number and 0, which needs no case of its own: a column of -inf alone ends
// with s = 0.
//
// Exponentials are the hardware's 2^z of the product with log2 e, within (|x - m|
// + 1) 2^-23 of themselves: the sum's small terms have the large errors, and an
// element of the gradient keeps its own in proportion (what is below 2^-126 may
// come out as zero).  An accurate one takes several instructions more, for which
// bf16 logits leave no room.
struct Stat {
    float m, s;
};
constexpr float GROW = 4.f;

__device__ __forceinline__ Stat stat_join(Stat a, Stat b) {
    const float m = fmaxf(a.m, b.m);
    return {m, a.s * __expf(a.m - m) + b.s * __expf(b.m - m)};
}

// n of them, `step` apart: the largest reference first, so that no exponential
// waits for another.
__device__ __forceinline__ Stat stat_join(const Stat *q, int n, int step) {
    Stat a = {-FLT_MAX, 0.f};
#pragma unroll 4
    for (int i = 0; i < n; ++i)
        a.m = fmaxf(a.m, q[i * step].m);
#pragma unroll 4
    for (int i = 0; i < n; ++i)
        a.s += q[i * step].s * __expf(q[i * step].m - a.m);
    return a;
}

// U rows of VEC columns into the columns' running (m, s).  The reference
// moves only when some value is GROW above it (the sums then rescale), so the
// usual group costs one exponential for each element and none besides, and
// one maximum over all its differences instead of one for each column.
template <int U, int VEC>
__device__ __forceinline__ void stat_add(const float (*x)[VEC], float *m, float *s) {
    float d[U][VEC], most = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            d[u][k] = x[u][k] - m[k];
            most = fmaxf(most, d[u][k]);
        }
    if (__any(most > GROW))
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            float top = m[k];
#pragma unroll
            for (int u = 0; u < U; ++u)
                top = fmaxf(top, x[u][k]);
            s[k] *= __expf(m[k] - top);
            m[k] = top;
#pragma unroll
            for (int u = 0; u < U; ++u)
                d[u][k] = x[u][k] - top;
        }
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        float sum = __expf(d[0][k]);
#pragma unroll
        for (int u = 1; u < U; ++u)
            sum += __expf(d[u][k]);
        s[k] += sum;
    }
}

// How the logits are cut.  FLAT (columns of a row fit the work-group):
// `lanes` threads, a multiple of the vectors after which columns repeat, walk
// a chunk's elements in one piece.  WIDE: a wave takes 64 * VEC columns of a
// row, the work-group's four waves every fourth row.
struct Cut {
    int T, V, B;
    int rows, chunks;  // rows of a chunk, chunks of a step
    int lanes;         // FLAT: threads at work; WIDE: 0
    int windows;       // WIDE: windows of 64 * VEC columns
    unsigned first;    // work-groups below it read the logits past the caches
    int mis;           // elements from the 16-byte boundary before the logits to their start
};

// A chunk's place: elements [lo, hi) counted from the 16-byte boundary.
struct Piece {
    int t, c, v0, v1;
    long lo, hi;
};

__device__ __forceinline__ Piece piece_of(const Cut &g, uint32_t block) {
    Piece p;
    p.t = (int)(block / (uint32_t)g.chunks);
    p.c = (int)(block - (uint32_t)p.t * g.chunks);
    p.v0 = p.c * g.rows;
    p.v1 = min(g.V, p.v0 + g.rows);
    const long s0 = (long)p.t * g.V * g.B + g.mis;
    p.lo = s0 + (long)p.v0 * g.B;
    p.hi = s0 + (long)p.v1 * g.B;
    return p;
}

// The column of element `at` (counted as in Piece, after lo - VEC and at most a
// work-group's vectors from there).
__device__ __forceinline__ int column_of(const Cut &g, const Piece &p, long at) {
    const int r = (int)(at - p.lo);
    return (uint32_t)(r + g.B * 16) % (uint32_t)g.B;
}

// f with std::true_type or std::false_type.
template <class F>
__device__ __forceinline__ void either(bool yes, F &&f) {
    if (yes)
        f(std::true_type());
    else
        f(std::false_type());
}

// VEC elements at `at`, those outside [lo, hi) -inf and not touched.
template <typename TS>
__device__ __forceinline__ void load_edge(const TS *x, long at, long lo, long hi, float *f) {
    constexpr int VEC = vec_of<TS>();
    if (at >= lo && at + VEC <= hi)
        load16(x + at, f);
    else
        load_part(x + at, (int)max(lo - at, 0L), (int)min(hi - at, (long)VEC), f, -INFINITY);
}

// (m, s) of a chunk's columns.  Bound by the memory and, in bf16, nearly by the
// exponentials: 410 MB in 78 us, most of it past the caches, where reading alone
// takes 58.
template <typename TS>
__global__ __launch_bounds__(NT) void stat_flat_kernel(Cut g, const TS *logits, Stat *stat) {
    constexpr int U = 4, VEC = vec_of<TS>();
    __shared__ Stat part[NT * VEC];
    const bool past = blockIdx.x < g.first;
    const Piece p = piece_of(g, blockIdx.x);
    const TS *x = logits - g.mis;
    const long first = p.lo / VEC * VEC;
    const int j = threadIdx.x;
    if (j < g.lanes) {
        const long step = (long)g.lanes * VEC;
        float m[VEC], s[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            m[k] = -FLT_MAX;
            s[k] = 0.f;
        }
        long at = first + (long)j * VEC;
        float f[U][VEC];
        if (at < p.lo) {
            load_edge(x, at, p.lo, p.hi, f[0]);
            stat_add<1, VEC>(f, m, s);
            at += step;
        }
        either(past, [&](auto how) {
            for (; at + (U - 1) * step + VEC <= p.hi; at += U * step) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    load16<how.value>(x + at + u * step, f[u]);
                stat_add<U, VEC>(f, m, s);
            }
        });
        for (; at < p.hi; at += step) {
            load_edge(x, at, p.lo, p.hi, f[0]);
            stat_add<1, VEC>(f, m, s);
        }
#pragma unroll
        for (int k = 0; k < VEC; ++k)
            part[j * VEC + k] = {m[k], s[k]};
    }
    __syncthreads();
    // entry q is of column (c0 + q) mod B: `n` entries of each, B apart, which
    // rounds of joins of four or more bring down to one
    const int c0 = column_of(g, p, first);
    for (int n = g.lanes * VEC / g.B; n > 1;) {
        const int left = max(1, min((int)blockDim.x / g.B, (n + 3) / 4));
        for (int b = j; b < g.B * left; b += blockDim.x) { // entries 0 .. left - 1 of every column
            Stat a = part[b];
            for (int i = b + left * g.B; i < n * g.B; i += left * g.B)
                a = stat_join(a, part[i]);
            part[b] = a;
        }
        n = left;
        __syncthreads();
    }
    for (int b = j; b < g.B; b += blockDim.x) {
        const int c = c0 + b; // the column of entry b
        stat[((long)p.t * g.chunks + p.c) * g.B + (c >= g.B ? c - g.B : c)] = part[b];
    }
}

// The same for rows wider than a work-group's vectors, as of one product for all
// steps: 1 x 32000 x 6400 bf16 85 us (4.8 TB/s), 1 x 32000 x 6399, whose vectors
// straddle lines, 139 (with the token kernel, on the same logits again: 73 and 123).
// Their gradients take 135 and 160.
template <typename TS>
__global__ __launch_bounds__(NT) void stat_wide_kernel(Cut g, const TS *logits, Stat *stat) {
    constexpr int U = 4, VEC = vec_of<TS>();
    __shared__ Stat part[NT * VEC];
    const bool past = blockIdx.x < g.first;
    const Piece p = piece_of(g, blockIdx.x / g.windows);
    const int lane = threadIdx.x & 63, row = threadIdx.x >> 6;
    const int b = ((int)(blockIdx.x % g.windows) * 64 + lane) * VEC, nb = min(VEC, g.B - b);
    float m[VEC], s[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        m[k] = -FLT_MAX;
        s[k] = 0.f;
    }
    if (nb > 0) {
        const TS *x = logits + (long)p.t * g.V * g.B + b;
        float f[U][VEC];
        int v = p.v0 + row;
        if (nb == VEC)
            either(past, [&](auto how) {
                for (; v + (U - 1) * 4 < p.v1; v += U * 4) {
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        load16<how.value>(x + (long)(v + u * 4) * g.B, f[u]);
                    stat_add<U, VEC>(f, m, s);
                }
            });
        for (; v < p.v1; v += 4) {
            if (nb == VEC)
                load16(x + (long)v * g.B, f[0]);
            else
                load_part(x + (long)v * g.B, 0, nb, f[0], -INFINITY);
            stat_add<1, VEC>(f, m, s);
        }
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k)
        part[(row * VEC + k) * 64 + lane] = {m[k], s[k]};
    __syncthreads();
    if (row == 0)
        for (int k = 0; k < nb; ++k)
            stat[((long)p.t * g.chunks + p.c) * g.B + b + k] = stat_join(part + k * 64 + lane, 4, VEC * 64);
}

// What the gradient kernel needs of a token: dL/dx_v = p * exp(min(x_v - m, GROW
// + 1)), m the reference that its sum s is of and p = -dlogp / s, and the
// gradient at the target itself.  m is a logit of the column, not m + log s: the
// difference is exact where the exponential counts, whatever the logits' size,
// where log s would be lost beside a large m.  A token that takes no part has p =
// 0: the minimum, which no other token meets (x_v is at most GROW above m), makes
// its exponentials finite whatever its logits are, so it gets zeros.
struct Coef {
    float m, p;
};

// What a token's terms are made of beside its column's (m, s): x is the
// target's logit.
struct TokenIn {
    int y;
    float x, w, old, ref, adv;
};

__device__ __forceinline__ TokenIn token_in(const LossArgs &a, int t, int b) {
    const long n = (long)t * a.B + b;
    TokenIn i = {a.targets[n], 0.f, 1.f, 0.f, 0.f, 0.f};
    if (a.weights)
        i.w = a.weights[n];
    if (a.old_logp)
        i.old = a.old_logp[n];
    if (a.ref_logp)
        i.ref = a.ref_logp[n];
    if (a.adv)
        i.adv = a.adv[n];
    if ((uint32_t)i.y < (uint32_t)a.V) {
        const long at = ((long)t * a.V + i.y) * a.B + b;
        i.x = a.bf16 ? st<bf16_t>::load((const bf16_t *)a.logits, at) : ((const float *)a.logits)[at];
    }
    return i;
}

// A token's logp, and what the gradient kernel needs of it, written; its loss
// term, in fp64.
__device__ __forceinline__ double token_terms(const LossArgs &a, Stat q, const TokenIn &i, long n, Coef *coef,
                                              float *dtarget) {
    double term = 0.0, lp = 0.0, g = 0.0;
    Coef c = {0.f, 0.f};
    float dt = 0.f;
    if ((uint32_t)i.y < (uint32_t)a.V && i.w != 0.f) {
        const double ls = log((double)q.s);
        lp = ((double)i.x - (double)q.m) - ls;
        if (a.mode == LOSS_XENT) {
            term = -lp;
            g = -1.0;
        } else if (a.mode == LOSS_POLICY) {
            const double A = i.adv;
            const double r = a.old_logp ? exp(lp - (double)i.old) : 1.0;
            const double cl = fmin(fmax(r, 1.0 - (double)a.clip_low), 1.0 + (double)a.clip_high);
            const double gain = r * A, held = cl * A;
            const bool open = gain <= held || gain != gain;
            term = -(open ? gain : held);
            g = open ? -gain : 0.0;
            if (a.ref_logp) {
                const double d = (double)i.ref - lp, e = expm1(d);
                term += (double)a.kl * (e - d);
                g -= (double)a.kl * e;
            }
        }
        term *= (double)i.w * (double)a.scale;
        g *= (double)i.w * (double)a.scale;
        if (g != 0.0) {
            c.m = q.m;
            c.p = (float)(-g / (double)q.s);
            dt = (float)(-g * expm1(lp));
        }
    }
    if (a.logp)
        a.logp[n] = (float)lp;
    coef[n] = c;
    dtarget[n] = dt;
    return term;
}

// 16 tokens to a work-group, 16 threads to a token: they join its chunks, and
// one of them does its terms in fp64, on operands read while the chunks were.
// Bound by latency: 4 us for 700 tokens, 5 for 6400.
constexpr int TOKENS = 16;

__global__ __launch_bounds__(NT) void token_kernel(LossArgs a, int chunks, const Stat *stat, Coef *coef, float *dtarget,
                                                   double *part) {
    constexpr int SUBS = NT / TOKENS, U = 4;
    __shared__ Stat join[NT / 64][TOKENS];
    const int j = threadIdx.x % TOKENS, sub = threadIdx.x / TOKENS;
    const long N = (long)a.T * a.B, n = (long)blockIdx.x * TOKENS + j;
    const int t = (int)(n / a.B), b = (int)(n - (long)t * a.B);
    TokenIn i = {-1};
    if (sub == 0 && n < N)
        i = token_in(a, t, b);
    Stat q = {-FLT_MAX, 0.f};
    if (n < N)
        for (int c = sub; c < chunks; c += SUBS * U) {
            Stat r[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                r[u] = c + u * SUBS < chunks ? stat[((long)t * chunks + c + u * SUBS) * a.B + b] : Stat{-FLT_MAX, 0.f};
            q = stat_join(q, stat_join(r, U, 1));
        }
#pragma unroll
    for (int m = TOKENS; m < 64; m <<= 1)
        q = stat_join(q, Stat{__shfl_xor(q.m, m, 64), __shfl_xor(q.s, m, 64)});
    if ((threadIdx.x & 63) < TOKENS)
        join[threadIdx.x >> 6][j] = q;
    __syncthreads();
    if (threadIdx.x >= TOKENS)
        return;
    double term = 0.0;
    if (n < N)
        term = token_terms(a, stat_join(&join[0][j], NT / 64, TOKENS), i, n, coef, dtarget);
#pragma unroll
    for (int m = TOKENS / 2; m >= 1; m >>= 1)
        term += __shfl_xor(term, m, 64);
    if (threadIdx.x == 0)
        part[blockIdx.x] = term;
}

// Sums and terms in one launch, for small logits: a work-group takes VEC columns
// of a step through all its rows.  The work-groups of a step read the same
// lines, so they go to one XCD (every eighth) while there are eight steps.
// Bound by latency: 1 x 10000 x 16 fp32 8.5 us.
constexpr int NARROW_NT = 1024;

template <typename TS>
__global__ __launch_bounds__(NARROW_NT) void narrow_kernel(LossArgs a, int groups, Coef *coef, float *dtarget, double *part) {
    constexpr int VEC = vec_of<TS>(), U = 32 / VEC, WAVES = NARROW_NT / 64, SUBS = WAVES / VEC;
    __shared__ Stat each[VEC][NARROW_NT];
    __shared__ Stat join[VEC][SUBS];
    int t, g;
    if (a.T >= 8) {
        const int q = blockIdx.x / 8;
        t = blockIdx.x % 8 + q / groups * 8;
        g = q % groups;
        if (t >= a.T)
            return;
    } else {
        t = blockIdx.x / groups;
        g = blockIdx.x % groups;
    }
    const int b0 = g * VEC, nb = min(VEC, a.B - b0), j = threadIdx.x;
    TokenIn in = {-1};
    if (j < nb)
        in = token_in(a, t, b0 + j);
    const TS *x = (const TS *)a.logits + (long)t * a.V * a.B + b0;
    float m[VEC], s[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        m[k] = -FLT_MAX;
        s[k] = 0.f;
    }
    for (int v = j; v < a.V; v += U * NARROW_NT) {
        float f[U][VEC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = v + u * NARROW_NT;
            if (r < a.V && nb == VEC)
                load16(x + (long)r * a.B, f[u]);
            else
                load_part(x + (long)r * a.B, 0, r < a.V ? nb : 0, f[u], -INFINITY);
        }
        stat_add<U, VEC>(f, m, s);
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k)
        each[k][j] = {m[k], s[k]};
    __syncthreads();
    // SUBS waves to a column
    {
        const int k = (j >> 6) % VEC, sub = (j >> 6) / VEC;
        Stat q = stat_join(&each[k][sub * 64 + (j & 63)], NARROW_NT / (64 * SUBS), 64 * SUBS);
        float top = q.m;
#pragma unroll
        for (int w = 32; w >= 1; w >>= 1)
            top = fmaxf(top, __shfl_xor(top, w, 64));
        float sum = q.s * __expf(q.m - top);
#pragma unroll
        for (int w = 32; w >= 1; w >>= 1)
            sum += __shfl_xor(sum, w, 64);
        if ((j & 63) == 0)
            join[k][sub] = {top, sum};
    }
    __syncthreads();
    if (j >= VEC)
        return;
    double term = 0.0;
    if (j < nb)
        term = token_terms(a, stat_join(join[j], SUBS, 1), in, (long)t * a.B + b0 + j, coef, dtarget);
#pragma unroll
    for (int w = VEC / 2; w >= 1; w >>= 1)
        term += __shfl_xor(term, w, 64);
    if (j == 0)
        part[t * groups + g] = term;
}

// The loss: the token kernel's partial sums in a fixed order, by one
// work-group.
struct LossOut {
    const double *part;
    int parts;
    float *loss; // NULL: not asked for
};

__device__ __forceinline__ void loss_sum(const LossOut &o) {
    __shared__ double red[NT / 64];
    double sum = 0.0;
    for (int i = threadIdx.x; i < o.parts; i += blockDim.x)
        sum += o.part[i];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1)
        sum += __shfl_xor(sum, m, 64);
    if ((threadIdx.x & 63) == 0)
        red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < (int)blockDim.x / 64; ++w)
            sum += red[w];
        *o.loss = (float)sum;
    }
}

__global__ __launch_bounds__(NT) void loss_sum_kernel(LossOut o) { loss_sum(o); }

__device__ __forceinline__ float grad_of(float x, Coef c) { return c.p * __expf(fminf(x - c.m, GROW + 1.f)); }

// The targets' own elements of a piece, written over what the softmax's term
// alone gave them (same work-group, after a barrier).
template <typename TS>
__device__ __forceinline__ void grad_targets(const Cut &g, const Piece &p, int b0, int b1, const int32_t *targets,
                                             const float *dtarget, TS *y) {
    for (int b = b0 + threadIdx.x; b < b1; b += blockDim.x) {
        const long n = (long)p.t * g.B + b;
        const int v = targets[n];
        if (v >= p.v0 && v < p.v1)
            st<TS>::store(y, ((long)p.t * g.V + v) * g.B + b, dtarget[n]);
    }
}

// The gradient of a piece.  Bound by the memory: 410 MB of bf16 logits, about
// half of them from the last-level cache, and 410 MB of gradient in 123 us (6.7
// TB/s).  PAST: it is streamed.
template <typename TS, bool PAST>
__global__ __launch_bounds__(NT) void grad_flat_kernel(Cut g, const TS *logits, TS *dlogits, const int32_t *targets,
                                                       const Coef *coef, const float *dtarget, LossOut o) {
    constexpr int U = 4, VEC = vec_of<TS>();
    if (o.loss && blockIdx.x == 0)
        loss_sum(o);
    const bool past = gridDim.x - 1 - blockIdx.x < g.first;
    const Piece p = piece_of(g, gridDim.x - 1 - blockIdx.x);
    const TS *x = logits - g.mis;
    TS *y = dlogits - g.mis;
    const long first = p.lo / VEC * VEC;
    const int j = threadIdx.x;
    if (j < g.lanes) {
        const long step = (long)g.lanes * VEC;
        long at = first + (long)j * VEC;
        Coef c[VEC];
        int b = column_of(g, p, at);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            c[k] = coef[(long)p.t * g.B + b];
            b = b + 1 == g.B ? 0 : b + 1;
        }
        float f[U][VEC];
        auto edge = [&] {
            load_edge(x, at, p.lo, p.hi, f[0]);
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                f[0][k] = grad_of(f[0][k], c[k]);
            if (at >= p.lo && at + VEC <= p.hi)
                store16(y + at, f[0]);
            else
                store_part(y + at, (int)max(p.lo - at, 0L), (int)min(p.hi - at, (long)VEC), f[0]);
            at += step;
        };
        if (at < p.lo)
            edge();
        either(past, [&](auto how) {
            for (; at + (U - 1) * step + VEC <= p.hi; at += U * step) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    load16<how.value>(x + at + u * step, f[u]);
#pragma unroll
                for (int u = 0; u < U; ++u) {
#pragma unroll
                    for (int k = 0; k < VEC; ++k)
                        f[u][k] = grad_of(f[u][k], c[k]);
                    store16<PAST>(y + at + u * step, f[u]);
                }
            }
        });
        while (at < p.hi)
            edge();
    }
    __syncthreads();
    grad_targets(g, p, 0, g.B, targets, dtarget, dlogits);
}

// PAST: the gradient is streamed.
template <typename TS, bool PAST>
__global__ __launch_bounds__(NT) void grad_wide_kernel(Cut g, const TS *logits, TS *dlogits, const int32_t *targets,
                                                       const Coef *coef, const float *dtarget, LossOut o) {
    constexpr int U = 4, VEC = vec_of<TS>();
    if (o.loss && blockIdx.x == 0)
        loss_sum(o);
    const bool past = gridDim.x - 1 - blockIdx.x < g.first;
    const Piece p = piece_of(g, (gridDim.x - 1 - blockIdx.x) / g.windows);
    const int lane = threadIdx.x & 63, row = threadIdx.x >> 6;
    const int w0 = (int)((gridDim.x - 1 - blockIdx.x) % g.windows) * 64 * VEC, b = w0 + lane * VEC, nb = min(VEC, g.B - b);
    if (nb > 0) {
        Coef c[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k)
            c[k] = k < nb ? coef[(long)p.t * g.B + b + k] : Coef{0.f, 0.f};
        const long s0 = (long)p.t * g.V * g.B + b;
        float f[U][VEC];
        int v = p.v0 + row;
        if (nb == VEC)
            either(past, [&](auto how) {
                for (; v + (U - 1) * 4 < p.v1; v += U * 4) {
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        load16<how.value>(logits + s0 + (long)(v + u * 4) * g.B, f[u]);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
#pragma unroll
                        for (int k = 0; k < VEC; ++k)
                            f[u][k] = grad_of(f[u][k], c[k]);
                        store16<PAST>(dlogits + s0 + (long)(v + u * 4) * g.B, f[u]);
                    }
                }
            });
        for (; v < p.v1; v += 4) {
            const long at = s0 + (long)v * g.B;
            if (nb == VEC)
                load16(logits + at, f[0]);
            else
                load_part(logits + at, 0, nb, f[0], 0.f);
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                f[0][k] = grad_of(f[0][k], c[k]);
            if (nb == VEC)
                store16(dlogits + at, f[0]);
            else
                store_part(dlogits + at, 0, nb, f[0]);
        }
    }
    __syncthreads();
    grad_targets(g, p, w0, min(g.B, w0 + 64 * VEC), targets, dtarget, dlogits);
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// A work-group's share of a step: PIECE bytes of logits or more, and whole
// multiples of PIECE where a number of rows comes to that.  Each of the first
// kernel's leaves (m, s) of every column, which costs it and the token kernel
// time: 512 of them, as many more as get 48 KB each, and 2048 at most (us of the
// whole loss with 2048, 1024 and 512 of them: 35 x 10000 x 20 fp32 23.0, 22.7, 22.2;
// 35 x 10000 x 64 bf16 33.2, 32.0, 32.2; 50 x 32000 x 128 bf16 200, 208, 203).
// The gradient's work-groups leave nothing, so finer ones only end more evenly.
// 50 x 32000 x 128 bf16, loss and gradient, us by the gradient's piece: 32 KB 205,
// 16 KB 200, 8 KB 238, 4 KB 310; of about 25 KB, not on such boundaries, 223.
constexpr long PIECE = 16384, SHARE = 3 * PIECE, GRAD_GROUPS = 1L << 22;

long stat_groups(int T, int B, int V, int es) {
    return std::max(512L, std::min(2048L, (long)T * V * B * es / SHARE));
}

// What of the logits the first kernel leaves in the last-level cache (256 MB)
// for the gradient: the last of them; what comes before is read past it, which
// is faster by a fifth. 50 x 32000 x 128 bf16 (410 MB), loss and gradient, in pieces
// of about 25 KB: 224 us; all of it through the cache 233, all past it 238.
constexpr long KEEP_BYTES = 224L << 20;

// The cut of logits whose elements have es bytes.
Cut cut_of(int T, int B, int V, int es, int mis, long groups) {
    const int VEC = 16 / es;
    Cut g = {T, V, B, V, 1, 0, 1, 0, mis};
    const int repeat = B / std::gcd(B, VEC);
    if (repeat <= NT)
        g.lanes = NT / repeat * repeat;
    else
        g.windows = (int)ceil_div(B, 64 * VEC);
    const long across = (long)T * g.windows;
    const long by_groups = ceil_div(groups, across), by_bytes = (long)V * B * es / g.windows / PIECE;
    long chunks = std::max(1L, std::min(std::min(by_groups, by_bytes), (long)V));
    g.rows = (int)ceil_div(V, chunks);
    const long even = PIECE / std::gcd(PIECE, (long)B * es);
    if (even <= g.rows)
        g.rows = (int)(ceil_div(g.rows, even) * even);
    g.chunks = (int)ceil_div(V, g.rows);
    const long blocks = across * g.chunks, keep = KEEP_BYTES / std::max(1L, (long)T * V * B * es / blocks);
    g.first = (unsigned)std::max(0L, blocks - keep);
    return g;
}

// Groups of columns of a step where narrow_kernel takes the logits, else 0.  A
// work-group needs two rounds of loads in fp32, one in bf16 at most, and what
// the L2 of an XCD gives its work-groups, whole lines, is limited, more so where
// a step's work-groups are spread over the XCDs.  us of the targets' logp with
// and without it: 1 x 10000 x 16 fp32 8.0, 8.8; 16 x 5000 x 16 6.5, 8.9; 100 x 10000 x 4
// 7.8, 8.8; 1 x 1000 x 256 bf16 6.6, 8.8; but 1 x 10000 x 64 fp32 9.5, 8.8, 1 x 5000 x 256
// 14.0, 8.8, 1 x 32000 x 16 11.3, 8.6, and 1 x 10000 x 16 bf16 10.1, 8.8.
int narrow_groups(int T, int B, int V, int es) {
    const long g = ceil_div(B, 16 / es), line = std::min(128L, (long)B * es);
    const bool rounds = V <= (es == 4 ? 16384 : 4096);
    const long most = T >= 8 ? 3L << 20 : 3L << 19;
    return rounds && T * g <= 1024 && ceil_div(T * g, 8) * V * line <= most ? (int)g : 0;
}

struct LossWs {
    Stat *stat;
    Coef *coef;
    float *dtarget;
    double *part;
    size_t bytes;
    int parts;
};

LossWs layout(void *ws, int T, int B, size_t chunks, int groups) {
    const size_t N = (size_t)T * B;
    char *p = (char *)ws;
    LossWs w;
    w.parts = groups ? T * groups : (int)((N + TOKENS - 1) / TOKENS);
    size_t at = 0;
    w.stat = (Stat *)(p + at);
    at += groups ? 0 : align256(N * chunks * sizeof(Stat));
    w.coef = (Coef *)(p + at);
    at += align256(N * sizeof(Coef));
    w.dtarget = (float *)(p + at);
    at += align256(N * sizeof(float));
    w.part = (double *)(p + at);
    at += align256((size_t)w.parts * 8);
    w.bytes = at;
    return w;
}

template <typename TS>
hipError_t run(const LossArgs &a, hipStream_t s) {
    constexpr int ES = st<TS>::bytes;
    const int mis = (int)((uintptr_t)a.logits / ES % vec_of<TS>());
    Cut g = cut_of(a.T, a.B, a.V, ES, mis, stat_groups(a.T, a.B, a.V, ES));
    const int groups = narrow_groups(a.T, a.B, a.V, ES);
    const LossWs w = layout(a.ws, a.T, a.B, g.chunks, groups);
    const TS *x = (const TS *)a.logits;
    TS *y = (TS *)a.dlogits;
    hipError_t e;
    const unsigned grid = (unsigned)((long)g.T * g.chunks * g.windows);
    const unsigned flat = (unsigned)(ceil_div(std::max(g.lanes, 1), 64) * 64);
    if (groups) {
        const unsigned steps = a.T >= 8 ? (unsigned)ceil_div(a.T, 8) * 8 : (unsigned)a.T;
        hipLaunchKernelGGL(narrow_kernel<TS>, dim3(steps * groups), dim3(NARROW_NT), 0, s, a, groups, w.coef, w.dtarget, w.part);
    } else {
        if (g.lanes)
            hipLaunchKernelGGL((stat_flat_kernel<TS>), dim3(grid), dim3(flat), 0, s, g, x, w.stat);
        else
            hipLaunchKernelGGL((stat_wide_kernel<TS>), dim3(grid), dim3(NT), 0, s, g, x, w.stat);
        if ((e = hipGetLastError()) != hipSuccess)
            return e;
        hipLaunchKernelGGL(token_kernel, dim3((unsigned)w.parts), dim3(NT), 0, s, a, g.chunks, w.stat, w.coef, w.dtarget,
                           w.part);
    }
    if ((e = hipGetLastError()) != hipSuccess)
        return e;
    const LossOut o = {w.part, w.parts, a.loss};
    if (!y) {
        if (a.loss)
            hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(NT), 0, s, o);
        return hipGetLastError();
    }
    g = cut_of(g.T, g.B, g.V, ES, mis, GRAD_GROUPS);
    const unsigned pieces = (unsigned)((long)g.T * g.chunks * g.windows);
    const bool past = (long)g.T * g.V * g.B * ES >= STREAM_BYTES;
    const auto kernel = g.lanes ? (past ? grad_flat_kernel<TS, true> : grad_flat_kernel<TS, false>)
                                : (past ? grad_wide_kernel<TS, true> : grad_wide_kernel<TS, false>);
    hipLaunchKernelGGL(kernel, dim3(pieces), dim3(g.lanes ? flat : NT), 0, s, g, x, y, a.targets, w.coef, w.dtarget, o);
    return hipGetLastError();
}

} // namespace

size_t loss_ws(int T, int B, int V, bool bf16) {
    const int es = bf16 ? 2 : 4;
    return layout(nullptr, T, B, (size_t)cut_of(T, B, V, es, 0, stat_groups(T, B, V, es)).chunks,
                  narrow_groups(T, B, V, es)).bytes;
}

hipError_t launch_loss(const LossArgs &a, hipStream_t s) {
    return a.bf16 ? run<bf16_t>(a, s) : run<float>(a, s);
}

} // namespace lstmss
