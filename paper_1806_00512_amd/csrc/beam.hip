// Beam search: one step's choice among beams and tokens, the states put in the
// order of the beams they come from, and the paths at the end.
//
//   score[s][k][v] = scores[s][k] + logits[v][s K + k] - log sum exp(logits[:, s K + k])
//   the K largest of a sequence's K V, ties to the lowest k V + v
//
// The logits are read once: the scan leaves, of each group of consecutive
// tokens of a column, its largest logit and the sum of exponentials below it.
// The K best tokens lie in the K best groups (a group that is not among them
// has K tokens before its own best: the others' bests, larger or equal and of
// a lower index), so the choice reads the groups' maxima and then K groups.
// Comparisons are of 64 bits: which of two is the larger is the result.
#include "head.h"
#include "vec.h"

#include <float.h>

namespace lstmss {

namespace {

constexpr int MOST_ENTRIES = 8192; // groups of a sequence's beams: what a work-group keeps in LDS
constexpr int LIST = 512;

// The power of two from K on.
__host__ __device__ constexpr int beams_shift(int K) {
    int b = 0;
    while (1 << b < K)
        ++b;
    return b;
}

// Tokens of a group, 2^result.
__host__ __device__ constexpr int rows_shift(int V, int K) {
    int b = 6;
    while ((((V - 1) >> b) + 1) << beams_shift(K) > MOST_ENTRIES)
        ++b;
    return b;
}

// A logit as the search takes it: NaN is a token that is not there, +inf the
// largest number.
__device__ __forceinline__ float clean(float x) { return x != x ? -INFINITY : fminf(x, FLT_MAX); }

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

struct Scan {
    int V, N, groups, rows; // rows of a group
    int cx;                 // lanes along the columns' vectors, the others along the rows
    int tiles;              // wavefronts along the columns
    float2 *groups_of;      // [groups][N]: largest logit, sum of exponentials below it
};

// A wavefront: a group of tokens, cx vectors of columns; 64 / cx lanes share a
// vector's rows, 8 of which are on their way at once.
//
// Exponentials are the hardware's, of fp32 differences from a reference of the
// lane's own that moves only when a logit is 8 above it; eight of them are added
// in fp32 and the eights in 64 bits, since terms of one size added to a large
// fp32 sum are rounded the same way each time (2^22 tokens, 32 beams: the sum's
// logarithm was off by 202 u, u = 2^-24).  Whatever V is, it is within u (25 + 2.3 d),
// d the distance below the largest logit, averaged by the softmax and at most ln
// V: a term's exponential 2 + 2.3 d, eight terms' sum 7, moves of the reference 4 (two
// of them leave nothing of 2^18 terms), the lane's factor 2 and two roundings, the
// lanes' sum 6, the group's factor 2 and a rounding.
//
// 32000 x 512 bf16 logits 15.5 us (7 us is their reading), 10000 x 4 in fp32 4.9 us:
// loads, then exponentials, then exchanges between lanes, with little to overlap.
template <typename TS>
__global__ void __launch_bounds__(256) beam_scan_kernel(const Scan a, const TS *x) {
    constexpr int VEC = vec_of<TS>(), AHEAD = 8;
    const int lane = threadIdx.x & 63, wave = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int group = wave / a.tiles, c = lane % a.cx, rl = 64 / a.cx;
    if (group >= a.groups)
        return;
    const int col = ((wave - group * a.tiles) * a.cx + c) * VEC;
    const int n = min(VEC, a.N - col); // columns that are there (0 or less: none)
    const int v0 = group * a.rows, v1 = min(a.V, v0 + a.rows);
    float m[VEC], ref[VEC]; // largest, reference of the sum
    double s[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        m[k] = ref[k] = -INFINITY;
        s[k] = 0.0;
    }
    if (n > 0)
        for (int v = v0 + lane / a.cx; v < v1; v += AHEAD * rl) {
            float f[AHEAD][VEC];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int at = v + i * rl;
                if (at >= v1) {
#pragma unroll
                    for (int k = 0; k < VEC; ++k)
                        f[i][k] = -INFINITY;
                } else if (n == VEC) {
                    load16(x + (long)at * a.N + col, f[i]);
                } else {
                    load_part(x + (long)at * a.N + col, 0, n, f[i], -INFINITY);
                }
            }
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                float top = m[k];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    f[i][k] = clean(f[i][k]);
                    top = fmaxf(top, f[i][k]);
                }
                m[k] = top;
                if (top > ref[k] + 8.f) {
                    s[k] *= exp_of(ref[k] - top);
                    ref[k] = top;
                }
                if (top > -INFINITY) {
                    float add = 0.f;
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i)
                        add += exp_of(f[i][k] - ref[k]);
                    s[k] += add;
                }
            }
        }
    float sum[VEC];
    for (int d = a.cx; d < 64; d *= 2)
#pragma unroll
        for (int k = 0; k < VEC; ++k)
            m[k] = fmaxf(m[k], shfl_xor_f32(m[k], d));
#pragma unroll
    for (int k = 0; k < VEC; ++k)
        sum[k] = ref[k] > -INFINITY ? (float)(s[k] * exp_of(ref[k] - m[k])) : 0.f;
    for (int d = a.cx; d < 64; d *= 2)
#pragma unroll
        for (int k = 0; k < VEC; ++k)
            sum[k] += shfl_xor_f32(sum[k], d);
    if (lane < a.cx)
#pragma unroll
        for (int k = 0; k < VEC; ++k)
            if (k < n)
                a.groups_of[(long)group * a.N + col + k] = float2{m[k], sum[k]};
}

struct Pick {
    int V, N, K, groups, eos;
    int kshift, rshift; // of a group's beams and of its rows
    const float *scores;
    const int32_t *done;
    const float2 *groups_of;
    float *scores_out;
    int32_t *tokens, *parents, *done_out;
};

// A candidate: its score's bits in the order of unsigned numbers, and its place
// (none: all ones, which nothing comes after).
struct Best {
    uint64_t key;
    uint32_t at;
};
constexpr Best NONE = {0, 0xffffffffu};

__device__ __forceinline__ Best candidate(double score, uint32_t at) {
    const uint64_t u = (uint64_t)__double_as_longlong(score + 0.0); // (-0 is 0)
    const uint64_t key = u ^ ((uint64_t)((int64_t)u >> 63) | 0x8000000000000000ull);
    const bool there = score > -INFINITY;
    return Best{there ? key : NONE.key, there ? at : NONE.at};
}

__device__ __forceinline__ double score_of(const Best &b) {
    const uint64_t u = b.key & 0x8000000000000000ull ? b.key ^ 0x8000000000000000ull : ~b.key;
    return __longlong_as_double((long long)u);
}

__device__ __forceinline__ bool before(const Best &a, const Best &b) {
    return (a.key > b.key) | ((a.key == b.key) & (a.at < b.at));
}

__device__ __forceinline__ Best first_of(Best b, int from, int to) {
    for (int d = from; d < to; d *= 2) {
        Best o;
        o.key = __shfl_xor((unsigned long long)b.key, d, 64);
        o.at = __shfl_xor(b.at, d, 64);
        const bool other = before(o, b);
        b.key = other ? o.key : b.key;
        b.at = other ? o.at : b.at;
    }
    return b;
}

struct Select {
    Best each[32];
    Best list[LIST];
    Best bound;
    int listed;
};

// The first two in order of a thread's entries.
struct Two {
    Best one = NONE, two = NONE;
    __device__ __forceinline__ void add(const Best &c) {
        const bool first = before(c, one), second = before(c, two);
        two.key = first ? one.key : second ? c.key : two.key;
        two.at = first ? one.at : second ? c.at : two.at;
        one.key = first ? c.key : one.key;
        one.at = first ? c.at : one.at;
    }
};

// The K first in order of n entries, into first[] (none past the last one); `own`:
// two of this thread's, which has the entries e = tid modulo the threads, with the
// largest keys (which of equal ones does not matter).
//
// Every TH / 32 threads find the first of their entries.  The K-th of these 32
// bounds what can be among the K first of all; what is not after it, a few more
// than K, is listed, and a listed entry's place is the number of those before it.
// (A thread looks at its entries again only where its second's key is not below
// the bound's either.)  Where the list overflows the first are found one after another,
// each by a search over all threads.
template <int TH, class Entry>
__device__ __forceinline__ void select_first(int n, int K, Select &s, Best *first, const Two &own, Entry &&entry) {
    const int tid = threadIdx.x, lane = tid & 63;
    const Best some = first_of(own.one, 1, TH / 32);
    if (tid == 0) {
        s.listed = 0;
        s.bound = NONE; // (fewer than K: all count)
    }
    if (tid < K)
        first[tid] = NONE;
    if (tid % (TH / 32) == 0)
        s.each[tid / (TH / 32)] = some;
    __syncthreads();
    if (tid < 64) {
        const Best c = s.each[lane & 31];
        const uint32_t lo = (uint32_t)c.key, hi = (uint32_t)(c.key >> 32);
        int place = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            Best o;
            o.key = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, i) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, i);
            o.at = __builtin_amdgcn_readlane(c.at, i);
            place += before(o, c);
        }
        if (lane < 32 && place == K - 1 && c.at != NONE.at)
            s.bound = c;
    }
    __syncthreads();
    const Best bound = s.bound;
    auto list = [&](const Best &b) {
        const int i = atomicAdd(&s.listed, 1);
        if (i < LIST)
            s.list[i] = b;
    };
    if (own.one.at != NONE.at && own.one.key >= bound.key) {
        if (own.two.at == NONE.at || own.two.key < bound.key) {
            if (!before(bound, own.one))
                list(own.one);
        } else {
            for (int e = tid; e < n; e += TH) {
                const Best b = entry(e);
                if (b.at != NONE.at && !before(bound, b))
                    list(b);
            }
        }
    }
    __syncthreads();
    const int m = s.listed;
    if (m <= LIST) {
        for (int i = tid; i < m; i += TH) {
            const Best b = s.list[i];
            int rank = 0;
#pragma unroll 4
            for (int q = 0; q < m; ++q)
                rank += before(s.list[q], b);
            if (rank < K)
                first[rank] = b;
        }
    } else {
        Best mine = NONE;
        for (int e = tid; e < n; e += TH) {
            const Best c = entry(e);
            if (before(c, mine))
                mine = c;
        }
        for (int j = 0; j < K; ++j) {
            const Best b = first_of(mine, 1, 64);
            __syncthreads();
            if (lane == 0)
                s.each[tid >> 6] = b;
            __syncthreads();
            Best last = s.each[0];
            for (int w = 1; w < TH / 64; ++w)
                if (before(s.each[w], last))
                    last = s.each[w];
            if (tid == 0)
                first[j] = last;
            if (mine.at == last.at && mine.at != NONE.at) { // (places are distinct: one thread's)
                mine = NONE;
                for (int e = tid; e < n; e += TH) {
                    const Best c = entry(e);
                    if (before(last, c) && before(c, mine))
                        mine = c;
                }
            }
        }
    }
    __syncthreads();
}

// A work-group chooses for one sequence.  Latency bound: 9 us for 157 groups of four
// beams, 13 us for 500 of eight (64 sequences at once), of which the groups' reading
// and the sums take about 3, each selection 2.
template <typename TS, int TH>
__global__ void __launch_bounds__(TH) beam_pick_kernel(const Pick a, const TS *x) {
    // of a beam: its score less the sum's logarithm, and its largest logit (from which
    // logits are taken: two of any size that are near each other keep their difference)
    __shared__ double base[32], most[32];
    __shared__ int over[32];
    __shared__ Best first[32], chosen[32];
    __shared__ Select sel;
    __shared__ float tops[MOST_ENTRIES], sums[MOST_ENTRIES]; // [groups][2^kshift]
    __shared__ float pm[TH / 64][32];
    __shared__ double ps[TH / 64][32];
    const int tid = threadIdx.x, K = a.K, kshift = a.kshift, kp = 1 << kshift;
    const long col0 = (long)blockIdx.x * K;
    const int k = tid & (kp - 1), r = tid >> kshift, step = TH >> kshift;
    const int lane = tid & 63, w = tid >> 6;

    // log sum exp of every beam; the two largest of a thread's groups, all of its beam k
    // (different logits can be equal scores, and the lowest group another than these)
    float top = -INFINITY, two = -INFINITY;
    int gtop = 0, gtwo = 0;
    const float2 *at = a.groups_of + col0 + k;
#pragma unroll 8
    for (int g = r; g < a.groups; g += step) {
        const float2 f = k < K ? at[(long)g * a.N] : float2{-INFINITY, 0.f};
        tops[(g << kshift) + k] = f.x;
        sums[(g << kshift) + k] = f.y;
        const bool first = f.x > top, second = f.x > two;
        two = first ? top : second ? f.x : two;
        gtwo = first ? gtop : second ? g : gtwo;
        top = first ? f.x : top;
        gtop = first ? g : gtop;
    }
    float all = top;
    for (int d = kp; d < 64; d *= 2)
        all = fmaxf(all, shfl_xor_f32(all, d));
    if (lane < kp)
        pm[w][lane] = all;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TH / 64; ++i)
        all = fmaxf(all, pm[i][k]);
    double s = 0.0;
    if (all > -INFINITY) {
#pragma unroll 4
        for (int g = r; g < a.groups; g += step)
            s += (double)(sums[(g << kshift) + k] * exp_of(tops[(g << kshift) + k] - all));
    }
    for (int d = kp; d < 64; d *= 2)
        s += shfl_xor_f64(s, d);
    if (lane < kp)
        ps[w][lane] = s;
    __syncthreads();
    if (tid < K) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < TH / 64; ++i)
            sum += ps[i][k];
        const bool fin = a.done && a.done[col0 + k] != 0;
        over[k] = fin;
        const double sc = (double)a.scores[col0 + k];
        // (a score that is NaN is a beam that is not there)
        base[k] = !(sc > -INFINITY) ? -INFINITY : fin ? sc : all > -INFINITY ? sc - log(sum) : -INFINITY;
        most[k] = all > -INFINITY ? all : 0.0;
    }
    __syncthreads();

    // the K best groups
    const int end = a.eos >= 0 ? a.eos >> a.rshift : -1;
    const bool fin = k < K && over[k];
    const double mine = k < K ? base[k] : -INFINITY, from = k < K ? most[k] : 0.0;
    auto group = [&](int g, float f) {
        const double score = fin ? (g == end ? mine : -INFINITY) : mine + ((double)f - from);
        return candidate(score, k * a.groups + g);
    };
    Two own;
    if (fin) {
        if (end % step == r) // (one of this thread's)
            own.add(group(end, 0.f));
    } else {
        own.add(group(gtop, top));
        own.add(group(gtwo, two));
    }
    select_first<TH>(a.groups << kshift, K, sel, chosen, own, [&](int e) { return group(e >> kshift, tops[e]); });

    // the K best tokens in them
    auto token = [&](int e) {
        const uint32_t group = chosen[e >> a.rshift].at;
        if (group == NONE.at)
            return NONE;
        const int kk = group / (uint32_t)a.groups, g = group - kk * a.groups;
        const int v = (g << a.rshift) + (e & ((1 << a.rshift) - 1));
        if (v >= a.V)
            return NONE;
        const double score = over[kk] ? (v == a.eos ? base[kk] : -INFINITY)
                                      : base[kk] + ((double)clean(st<TS>::load(x, (long)v * a.N + col0 + kk)) - most[kk]);
        return candidate(score, (uint32_t)kk * a.V + v);
    };
    own = Two();
    for (int e = tid; e < K << a.rshift; e += TH)
        own.add(token(e));
    select_first<TH>(K << a.rshift, K, sel, first, own, token);
    if (tid < K) {
        const Best b = first[tid];
        const bool there = b.at != NONE.at;
        const int parent = there ? b.at / (uint32_t)a.V : tid, token = there ? (int)(b.at - (uint32_t)parent * a.V) : -1;
        a.scores_out[col0 + tid] = there ? (float)score_of(b) : -INFINITY;
        a.tokens[col0 + tid] = token;
        a.parents[col0 + tid] = parent;
        if (a.done_out)
            a.done_out[col0 + tid] = there && (over[parent] || token == a.eos);
    }
}

// out[r][s K + k] = x[r][s K + parents[s K + k]]; zero where the parent is no beam.
// Memory bound: 33 MB of states in 12 to 19 us.
template <typename T>
__global__ void __launch_bounds__(256) beam_reorder_kernel(long rows, int N, int K, const int32_t *parents, const T *x,
                                                           T *out) {
    const int col = blockIdx.x * 256 + threadIdx.x;
    if (col >= N)
        return;
    const int p = parents[col];
    const bool there = p >= 0 && p < K;
    const int from = col - col % K + (there ? p : 0);
    for (long r = blockIdx.y; r < rows; r += gridDim.y)
        out[r * N + col] = there ? x[r * N + from] : T(0);
}

// The tokens on the way to every beam: a thread walks back from one.
__global__ void __launch_bounds__(256) beam_trace_kernel(int T, int N, int K, const int32_t *tokens,
                                                         const int32_t *parents, int32_t *out) {
    const int col = blockIdx.x * 256 + threadIdx.x;
    if (col >= N)
        return;
    const int first = col - col % K;
    int at = col;
    for (int t = T - 1; t >= 0; --t) {
        const long i = (long)t * N;
        out[i + col] = at < 0 ? -1 : tokens[i + at];
        if (at >= 0) {
            const int p = parents[i + at];
            at = p >= 0 && p < K ? first + p : -1;
        }
    }
}

int groups_of(int V, int K) { return ((V - 1) >> rows_shift(V, K)) + 1; }

template <typename TS>
hipError_t beam_typed(const BeamArgs &a, hipStream_t s) {
    constexpr int VEC = vec_of<TS>();
    const int N = a.S * a.K;
    Scan c;
    c.V = a.V;
    c.N = N;
    c.rows = 1 << rows_shift(a.V, a.K);
    c.groups = groups_of(a.V, a.K);
    c.cx = 1;
    while (c.cx * VEC < N && c.cx < 8)
        c.cx *= 2;
    c.tiles = (int)ceil_div(N, c.cx * VEC);
    c.groups_of = (float2 *)a.ws;
    beam_scan_kernel<TS><<<dim3((unsigned)ceil_div((long)c.groups * c.tiles, 4)), 256, 0, s>>>(c, (const TS *)a.logits);
    Pick p;
    p.V = a.V;
    p.N = N;
    p.K = a.K;
    p.groups = c.groups;
    p.kshift = beams_shift(a.K);
    p.rshift = rows_shift(a.V, a.K);
    p.eos = a.eos;
    p.scores = a.scores;
    p.done = a.done;
    p.groups_of = c.groups_of;
    p.scores_out = a.scores_out;
    p.tokens = a.tokens;
    p.parents = a.parents;
    p.done_out = a.done_out;
    // threads: few groups are quicker with few (a barrier is of fewer wavefronts)
    if ((c.groups << p.kshift) <= 2048)
        beam_pick_kernel<TS, 256><<<dim3(a.S), 256, 0, s>>>(p, (const TS *)a.logits);
    else
        beam_pick_kernel<TS, 1024><<<dim3(a.S), 1024, 0, s>>>(p, (const TS *)a.logits);
    return hipGetLastError();
}

} // namespace

size_t beam_ws(int S, int K, int V) { return (size_t)groups_of(V, K) * S * K * 8; }

hipError_t launch_beam(const BeamArgs &a, hipStream_t s) {
    return a.bf16 ? beam_typed<bf16_t>(a, s) : beam_typed<float>(a, s);
}

hipError_t launch_beam_reorder(long rows, int N, int K, bool bf16, const int32_t *parents, const void *x, void *out,
                               hipStream_t s) {
    const dim3 grid((unsigned)ceil_div(N, 256), (unsigned)(rows < 4096 ? rows : 4096));
    if (bf16)
        beam_reorder_kernel<<<grid, 256, 0, s>>>(rows, N, K, parents, (const uint16_t *)x, (uint16_t *)out);
    else
        beam_reorder_kernel<<<grid, 256, 0, s>>>(rows, N, K, parents, (const float *)x, (float *)out);
    return hipGetLastError();
}

hipError_t launch_beam_trace(int T, int N, int K, const int32_t *tokens, const int32_t *parents, int32_t *out,
                             hipStream_t s) {
    beam_trace_kernel<<<dim3((unsigned)ceil_div(N, 256)), 256, 0, s>>>(T, N, K, tokens, parents, out);
    return hipGetLastError();
}

} // namespace lstmss
