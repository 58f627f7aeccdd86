// Embedding lookup into the batch-last layout, and its gradient by sorted
// tokens.
//
// Lookup: x[t][i][b] = scale * E[tokens[t][b]][i].  The table has its features
// in one piece, x its batch: a work-group reads 64 features of up to 64
// columns' rows, turns them over in LDS and writes them batch-last.  Bound by
// the memory (the rows in use read, x written), with dropout on bf16 also by
// Philox.  100 x 256 tokens of a Zipf law, 4096 features, 32000 rows, three sets
// of tokens in turn: bf16 57 us (210 MB written, about 60 MB of rows: 4.8 TB/s),
// with dropout 68; fp32 132 and 142.  The same tokens again, whose rows are then in
// the last-level cache: 44, 57; 84, 90.  A batch that is no multiple of 64 takes
// the kernel's general form: 100 x 255 tokens, 4095 features, bf16 with dropout
// 191 us, and 407 with a mask that repeats after no multiple of 8.
//
// Gradient: dE[v][i] = scale * sum of dX[t][i][b] over the (t, b) with token v.
//   sort_kernel   the positions' ranks by (token, position), and each token's
//                 range of ranks; dE is zeroed by the same launch
//   turn_kernel   dX turned over as in the lookup, each position's row written
//                 at its rank (the row of a token that stands once goes
//                 straight into dE)
//   walk_kernel   sums of equal tokens' rows, which now follow one another, over
//                 groups of rows
//   carry_kernel  tokens whose rows lie in several groups
// (few positions: sort_kernel and few_kernel alone).  The order of every sum
// follows from the tokens alone.  Bound by the memory: 50 x 128 tokens, 2048
// features, 32000 rows 83 us (dE 262 MB written, dX 52 MB read: 3.8 TB/s; the
// sort with the zeroing 48 us, the turn 21, the walk 9, the carry 5), added to dE
// 49 (10, 24, 11, 4); 35 x 20 tokens, 650 features, 10000 rows 12 us, two launches
// of 7 and 6.  The sort is what grows with N * V: see there.
#include <algorithm>

#include "common.h"
#include "language.h"
#include "philox.h"
#include "vec.h"

namespace lstmss {

namespace {

constexpr int NT = 256;
constexpr int TILE = 64;        // features and columns of a tile
constexpr int PITCH = TILE + 1; // its columns' distance in LDS: both ways of access meet all banks alike

// A step's columns are cut into chunks of `cols` (one chunk: cols = B), its
// features into tiles of 64.  With one chunk a tile of the batch-last tensor
// is one piece of memory, else it is a piece for each feature.
struct Tiling {
    int T, B, I;
    int cols, chunks, tiles;
};

struct Tile {
    int t, b0, nb, i0, ni;
};

__device__ __forceinline__ Tile tile_of(const Tiling &g, long block) {
    Tile a;
    const long tc = block / g.tiles;
    a.i0 = (int)(block - tc * g.tiles) * TILE;
    a.t = (int)(tc / g.chunks);
    a.b0 = (int)(tc - (long)a.t * g.chunks) * g.cols;
    a.nb = min(g.cols, g.B - a.b0);
    a.ni = min(TILE, g.I - a.i0);
    return a;
}

// Calls f(e, lo, hi, i, b, whole) for the groups of VEC elements (16 bytes) from
// e, a multiple of VEC, that cover a tile of the batch-last tensor, those in [lo, hi)
// its own: element e + k is of column b + k, feature i while b + k < B, of the
// next features from there.  b may be negative, above -VEC, in a group that
// begins before its piece.  `whole` holds for a group that is its tile's alone
// and of one feature, which all are where B is a multiple of VEC.
template <int VEC, class F>
__device__ __forceinline__ void for_groups(const Tiling &g, const Tile &a, F &&f) {
    if (g.chunks == 1) {
        const long lo = ((long)a.t * g.I + a.i0) * g.B, hi = lo + (long)a.ni * g.B;
        const long q0 = lo / VEC, q1 = (hi + VEC - 1) / VEC;
        for (long q = q0 + threadIdx.x; q < q1; q += NT) {
            const int r = (int)(q * VEC - lo);
            const int i = r < 0 ? 0 : r / g.B, b = r - i * g.B;
            f(q * VEC, lo, hi, i, b, r >= 0 && q * VEC + VEC <= hi && b + VEC <= g.B);
        }
    } else {
        const int per = (a.nb + VEC - 1) / VEC + 1;
        for (int n = threadIdx.x; n < per * a.ni; n += NT) {
            const int i = n / per, j = n - i * per;
            const long lo = ((long)a.t * g.I + a.i0 + i) * g.B + a.b0, hi = lo + a.nb;
            const long e = lo / VEC * VEC + j * VEC;
            if (e < hi)
                f(e, lo, hi, i, (int)(e - lo), e >= lo && e + VEC <= hi);
        }
    }
}

// Calls f(e, i, b) for the groups of a tile of 64 whole columns, each of one
// feature alone.
template <int VEC, class F>
__device__ __forceinline__ void for_whole_groups(const Tiling &g, const Tile &a, F &&f) {
    const long lo = ((long)a.t * g.I + a.i0) * g.B + a.b0;
    constexpr int PER = TILE / VEC;
    const int b = threadIdx.x % PER * VEC;
#pragma unroll
    for (int n = 0; n < TILE * PER / NT; ++n) {
        const int i = threadIdx.x / PER + n * (NT / PER);
        if (i < a.ni)
            f(lo + i * g.B + b, i, b);
    }
}

// A tile's elements, scaled and with dropout, from LDS to x.
template <bool PAST, typename TS>
__device__ __forceinline__ void write_tile(const EmbedArgs &a, const Tiling &g, const Tile &w, const float *tile, TS *x) {
    constexpr int VEC = vec_of<TS>();
    for_groups<VEC>(g, w, [&](long e, long lo, long hi, int i, int b, bool whole) {
        float f[VEC];
        if (whole) {
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                f[k] = tile[(b + k) * PITCH + i] * a.scale;
        } else {
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                f[k] = e + k >= lo && e + k < hi ? tile[b * PITCH + i] * a.scale : 0.f;
                if (++b == g.B) {
                    b = 0;
                    ++i;
                }
            }
        }
        drop_any<VEC>(a.drop, e, f);
        if (e >= lo && e + VEC <= hi)
            store16<PAST>(x + e, f);
        else
            store_part(x + e, (int)max(lo - e, 0L), (int)min(hi - e, (long)VEC), f);
    });
}

// A work-group's columns and `run` feature tiles one after the other: the next
// tile's rows are on their way while this one is turned over and written
// (4096 bf16 features, us: 79 and, with dropout, 92 so, 85 and 107 without; x was
// not streamed then).
// WHOLE: B is a multiple of 64, and the mask repeats after a multiple of 8 if
// at all; DROP: with dropout (only told apart there).  PAST: x is streamed.
template <typename TS, bool WHOLE, bool DROP, bool PAST>
__global__ __launch_bounds__(NT) void embed_kernel(EmbedArgs a, Tiling g, int run) {
    constexpr int LV = vec_of<TS>(), PER = TILE / LV, LOADS = TILE * PER / NT;
    __shared__ float tile[TILE * PITCH];
    const int runs = (g.tiles + run - 1) / run;
    const int part = blockIdx.x % runs;
    const long steps = blockIdx.x / runs;
    const int last = min(g.tiles, (part + 1) * run);
    Tile w = tile_of(g, steps * g.tiles + part * run);
    const TS *row[LOADS];
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
        const int b = (threadIdx.x + k * NT) / PER;
        const int v = b < w.nb ? a.tokens[(long)w.t * g.B + w.b0 + b] : -1;
        row[k] = (uint32_t)v < (uint32_t)a.V ? (const TS *)a.E + (long)v * g.I : nullptr;
    }
    float f[LOADS][LV];
    const int i = threadIdx.x % PER * LV;
    auto fetch = [&](int i0) {
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            if (row[k] && i0 + i + LV <= g.I)
                load16(row[k] + i0 + i, f[k]);
            else
                load_part(row[k] + i0 + i, 0, row[k] ? g.I - i0 - i : 0, f[k], 0.f);
        }
    };
    fetch(w.i0);
    TS *x = (TS *)a.x;
    for (int n = part * run; n < last; ++n) {
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            const int b = (threadIdx.x + k * NT) / PER;
#pragma unroll
            for (int j = 0; j < LV; ++j)
                tile[b * PITCH + i + j] = f[k][j];
        }
        __syncthreads();
        w.i0 = n * TILE;
        w.ni = min(TILE, g.I - w.i0);
        if (n + 1 < last)
            fetch(w.i0 + TILE);
        if constexpr (WHOLE) {
            constexpr int VEC = vec_of<TS>();
            for_whole_groups<VEC>(g, w, [&](long e, int i, int b) {
                float o[VEC];
#pragma unroll
                for (int k = 0; k < VEC; ++k)
                    o[k] = tile[(b + k) * PITCH + i] * a.scale;
                if (DROP)
                    drop_whole<VEC>(a.drop, e, o);
                store16<PAST>(x + e, o);
            });
        } else
            write_tile<PAST>(a, g, w, tile, x);
        __syncthreads();
    }
}

// ------------------------------------------------------------ gradient

constexpr int SORT_NT = 1024, SORT_WAVES = SORT_NT / 64, SORT_MOST = 512;

constexpr long FILL = 16384; // elements that a work-group zeroes

__device__ __forceinline__ void zero_fill(float *p, long i0, long i1) {
    const float zero[4] = {};
    for (long i = i0 + threadIdx.x * 4; i < i1; i += SORT_NT * 4) {
        if (i + 4 <= i1)
            store16(p + i, zero);
        else
            store_part(p + i, 0, (int)(i1 - i), zero);
    }
}

// Work-group w places the tokens [w R, (w + 1) R): every wave counts its share
// of the positions by token; the counts before a (wave, token), with those of
// all smaller tokens, are where that wave's first position of the token goes,
// and the waves then go over their shares again in order.  Every work-group
// reads all tokens twice, which lie in the caches; none waits for another.  So a
// small call is bound by latency, and the time of a large one grows with N * V / R:
// without zeroing 5 us for 700 tokens of 10000 rows, 10 for 6400 of 32000, 45 for
// 25600 of 1000000, 1225 for 2^20 of 2^20 (the call's other kernels: 240, for 64
// features).
// The work-groups from `sorters` on zero dE meanwhile, which the sort leaves
// the memory free for: rows in use are written after this launch.  That hides
// the sort where dE is what takes longer (6400 tokens, 262 MB: 48 us), not where
// N * V is (25600 tokens, 32 MB: 48).
__global__ __launch_bounds__(SORT_NT) void sort_kernel(const int32_t *tokens, int N, int V, int R, int32_t *rank,
                                                       int32_t *order, int32_t *key, int32_t *start, int sorters,
                                                       float *dE, long size) {
    if ((int)blockIdx.x >= sorters) {
        const long i0 = (long)(blockIdx.x - sorters) * FILL, i1 = min(size, i0 + FILL);
        return zero_fill(dE, i0, i1);
    }
    __shared__ int hist[SORT_WAVES][SORT_MOST];
    __shared__ int less[SORT_WAVES], sums[SORT_WAVES];
    const int lo = blockIdx.x * R, n = min(V - lo, R);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int k = lane; k < R; k += 64)
        hist[w][k] = 0;
    __syncthreads();
    const int share = (int)(ceil_div(N, SORT_NT) * 64);
    const int p0 = (int)min((long)N, (long)w * share), p1 = (int)min((long)N, (long)p0 + share);
    // loads on their way together: 25600 positions, 8 features, 1000000 rows 66 us
    // so, 168 one by one, 68 by eights; 700 and 10000 rows alike, but 0.5 slower by eights
    constexpr int U = 4;
    int before = 0;
    for (int p = p0 + lane; p < p1; p += 64 * U) {
        uint32_t v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            v[u] = p + u * 64 < p1 ? (uint32_t)tokens[p + u * 64] : ~0u;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            before += v[u] < (uint32_t)lo;
            if (v[u] - (uint32_t)lo < (uint32_t)n)
                atomicAdd(&hist[w][v[u] - lo], 1);
        }
    }
    for (int m = 32; m >= 1; m >>= 1)
        before += __shfl_xor(before, m, 64);
    if (lane == 0)
        less[w] = before;
    __syncthreads();
    int at = 0;
    for (int k = 0; k < SORT_WAVES; ++k)
        at += less[k];
    // exclusive sums over the tokens (one for each of the first 512 threads), then over the waves
    int total = 0;
    if ((int)threadIdx.x < n)
        for (int k = 0; k < SORT_WAVES; ++k)
            total += hist[k][threadIdx.x];
    int sum = total;
    for (int m = 1; m < 64; m <<= 1) {
        const int o = __shfl_up(sum, m, 64);
        sum += lane >= m ? o : 0;
    }
    if (lane == 63)
        sums[w] = sum;
    __syncthreads();
    for (int k = 0; k < w; ++k)
        sum += sums[k];
    if ((int)threadIdx.x < n) {
        int first = at + sum - total;
        start[lo + threadIdx.x] = first;
        if (lo + (int)threadIdx.x == V - 1)
            start[V] = first + total;
        for (int k = 0; k < SORT_WAVES; ++k) {
            const int c = hist[k][threadIdx.x];
            hist[k][threadIdx.x] = first;
            first += c;
        }
    }
    __syncthreads();
    // 64 positions at once: the lanes with a lane's token are those that agree
    // with it in every bit of the token's place in the range
    volatile int *next = hist[w];
    const int bits = 32 - __clz(R - 1);
    const uint64_t below = (1ull << lane) - 1;
    for (int base = p0; base < p1; base += 64 * U) {
        uint32_t v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = base + u * 64 + lane;
            v[u] = p < p1 ? (uint32_t)tokens[p] : ~0u;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t k = v[u] - (uint32_t)lo;
            const bool in = k < (uint32_t)n;
            uint64_t same = __ballot(in);
            if (same == 0)
                continue;
            for (int j = 0; j < bits; ++j) {
                const uint64_t one = __ballot(k >> j & 1);
                same &= k >> j & 1 ? one : ~one;
            }
            if (in) {
                const int p = base + u * 64 + lane, first = next[k], r = first + __popcll(same & below);
                rank[p] = r;
                order[r] = p;
                key[r] = lo + (int)k;
                if ((same & below) == 0)
                    next[k] = first + __popcll(same);
            }
        }
    }
}

// A token's range of ranks.
struct Sorted {
    const int32_t *rank, *order, *key, *start; // [N], [N], [N], [V + 1]
};

__device__ __forceinline__ void put(const EmbedGradArgs &a, float *p, float sum) {
    *p = a.accumulate ? *p + sum * a.scale : sum * a.scale;
}

// A tile of dX, with dropout, into LDS.
__device__ __forceinline__ void turn_in(const EmbedGradArgs &a, const Tiling &g, const Tile &w, float *tile) {
    for_groups<4>(g, w, [&](long e, long lo, long hi, int i, int b, bool whole) {
        float f[4];
        if (e >= lo && e + 4 <= hi)
            load16(a.dX + e, f);
        else
            load_part(a.dX + e, (int)max(lo - e, 0L), (int)min(hi - e, 4L), f, 0.f);
        drop_any<4>(a.drop, e, f);
        if (whole) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                tile[(b + k) * PITCH + i] = f[k];
            return;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (e + k >= lo && e + k < hi)
                tile[b * PITCH + i] = f[k];
            if (++b == g.B) {
                b = 0;
                ++i;
            }
        }
    });
}

// WHOLE, DROP as for the lookup.  Bound by the memory: 52 MB of dX read and 45 MB
// of rows written in 21 us.  A work-group's columns and `run` feature
// tiles one after the other, the next tile's elements on their way meanwhile
// (WHOLE).
template <bool WHOLE, bool DROP>
__global__ __launch_bounds__(NT) void turn_kernel(EmbedGradArgs a, Tiling g, Sorted q, float *rows, int run) {
    constexpr int PER = TILE / 4, LOADS = TILE * PER / NT;
    __shared__ float tile[TILE * PITCH];
    __shared__ float *dest[TILE];
    __shared__ bool once[TILE];
    const int runs = (g.tiles + run - 1) / run;
    const int part = blockIdx.x % runs, last = min(g.tiles, (part + 1) * run);
    Tile w = tile_of(g, (long)(blockIdx.x / runs) * g.tiles + part * run);
    float f[LOADS][4];
    const int b = threadIdx.x % PER * 4;
    auto fetch = [&](int i0) {
        const long lo = ((long)w.t * g.I + i0) * g.B + w.b0 + b;
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            const int i = threadIdx.x / PER + k * (NT / PER);
            if (i0 + i < g.I)
                load16<true>(a.dX + lo + i * g.B, f[k]);
        }
    };
    if (WHOLE)
        fetch(w.i0);
    if ((int)threadIdx.x < w.nb) {
        const long p = (long)w.t * g.B + w.b0 + threadIdx.x;
        const int v = a.tokens[p];
        float *d = nullptr;
        bool one = false;
        if ((uint32_t)v < (uint32_t)a.V) {
            one = q.start[v + 1] - q.start[v] == 1;
            d = one ? a.dE + (long)v * a.I : rows + (long)q.rank[p] * a.I;
        }
        dest[threadIdx.x] = d;
        once[threadIdx.x] = one;
    }
    const int lane = threadIdx.x & 63;
    for (int n = part * run; n < last; ++n) {
        w.i0 = n * TILE;
        w.ni = min(TILE, g.I - w.i0);
        if constexpr (WHOLE) {
#pragma unroll
            for (int k = 0; k < LOADS; ++k) {
                const int i = threadIdx.x / PER + k * (NT / PER);
                if (i >= w.ni)
                    continue;
                if (DROP)
                    drop_whole<4>(a.drop, ((long)w.t * g.I + w.i0 + i) * g.B + w.b0 + b, f[k]);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    tile[(b + j) * PITCH + i] = f[k][j];
            }
        } else {
            turn_in(a, g, w, tile);
        }
        __syncthreads();
        if (WHOLE && n + 1 < last)
            fetch(w.i0 + TILE);
        if (lane < w.ni)
            for (int c = threadIdx.x >> 6; c < w.nb; c += NT / 64) {
                float *d = dest[c];
                if (!d)
                    continue;
                d += w.i0 + lane;
                if (once[c])
                    put(a, d, tile[c * PITCH + lane]);
                else
                    *d = tile[c * PITCH + lane];
            }
        __syncthreads();
    }
}

// Rows [G q, G q + G) of the sorted rows, four features to a thread: the sums
// of runs of equal tokens.  A run that begins and ends here is finished; what
// continues from the group before goes to carry[q][0], what begins here and
// goes on to carry[q][1].  6400 rows of 2048 features, us with groups of 16: 9; of
// 64, which leave too few work-groups, 23.
template <int G>
__global__ __launch_bounds__(NT) void walk_kernel(EmbedGradArgs a, Sorted q, const float *rows, float *carry, int parts) {
    constexpr int U = 8, VEC = 4;
    __shared__ int key[G + 2];
    const int group = blockIdx.x / parts, part = blockIdx.x - group * parts;
    const int M = q.start[a.V];
    const long r0 = (long)group * G;
    if (r0 >= M)
        return;
    const int n = (int)min((long)G, M - r0);
    for (int k = threadIdx.x; k < n + 2; k += NT) {
        const long r = r0 + k - 1;
        key[k] = r >= 0 && r < M ? q.key[r] : -1;
    }
    __syncthreads();
    const int i = (part * NT + threadIdx.x) * VEC;
    const int ni = min(VEC, a.I - i);
    if (ni <= 0)
        return;
    auto load = [&](const float *p, float *f) {
        if (ni == VEC)
            load16(p, f);
        else
            load_part(p, 0, ni, f, 0.f);
    };
    auto store = [&](float *p, const float *f) {
        if (ni == VEC)
            store16(p, f);
        else
            store_part(p, 0, ni, f);
    };
    float sum[VEC] = {};
    bool begun = key[0] != key[1]; // the run at hand begins in this group
    for (int k0 = 0; k0 < n; k0 += U) {
        float f[U][VEC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u;
            // a row whose token stands once is not there
            if (k < n && (key[k] == key[k + 1] || key[k + 1] == key[k + 2]))
                load(rows + (r0 + k) * a.I + i, f[u]);
            else
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    f[u][j] = 0.f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u;
            if (k >= n)
                break;
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                sum[j] += f[u][j];
            const int v = key[k + 1];
            const bool ends = v != key[k + 2];
            if (!ends && k + 1 < n)
                continue;
            if (begun && ends) {
                if (v != key[k]) {
                    // stands once: written already
                } else {
                    float *p = a.dE + (long)v * a.I + i;
                    float out[VEC] = {};
                    if (a.accumulate)
                        load(p, out);
#pragma unroll
                    for (int j = 0; j < VEC; ++j)
                        out[j] = a.accumulate ? out[j] + sum[j] * a.scale : sum[j] * a.scale;
                    store(p, out);
                }
            } else {
                store(carry + ((long)group * 2 + (begun ? 1 : 0)) * a.I + i, sum);
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                sum[j] = 0.f;
            begun = true;
        }
    }
}

// The run that crosses into group q from where it begins, in group q - 1: the
// sums of its parts, in order.
__global__ __launch_bounds__(NT) void carry_kernel(EmbedGradArgs a, Sorted s, const float *carry, int G, int parts) {
    const int q = blockIdx.x / parts + 1, part = blockIdx.x - (q - 1) * parts;
    const long r = (long)q * G;
    if (r >= s.start[a.V] || s.key[r - 1] != s.key[r])
        return;
    const int v = s.key[r];
    if (s.start[v] < r - G)
        return; // begins before group q - 1
    const int i = part * NT + threadIdx.x;
    if (i >= a.I)
        return;
    const int last = (s.start[v + 1] - 1) / G;
    const float first = carry[((long)(q - 1) * 2 + 1) * a.I + i];
    put(a, a.dE + (long)v * a.I + i, sum_parts(first, carry + (long)q * 2 * a.I + i, last - q + 1, 2L * a.I));
}

// Few positions: a work-group takes FEW features of all of them into LDS and
// sums there, a thread for each feature of a run; one launch instead of three.
// us, Zipf tokens over 5000 rows, this kernel with 4 and 8 features against the
// three launches: 992 positions, 1024 features 14.2, 15.7, 21.4; 2048 positions,
// 1024 features 21.3, 22.3, 25.2, 2048 features 31.0, 24.1, 28.5, 4096 features
// 50, 39, 36; 3968 positions, 1024 features 32, 40, 29.  So: 4 features while
// that makes no more work-groups than CUs; not over 2048 positions or 2^22
// elements.
constexpr int FEW_NT = 1024, FEW_MOST = 2048, FEW_CUS = 256;
constexpr long FEW_SIZE = 1L << 22;

template <int FEW>
constexpr size_t few_lds(int N) {
    return (size_t)N * ((FEW + 1) * sizeof(float) + sizeof(int32_t) + 2 * sizeof(uint16_t));
}

template <int FEW>
__global__ __launch_bounds__(FEW_NT) void few_kernel(EmbedGradArgs a, Sorted q, int N) {
    constexpr int FEW_PITCH = FEW + 1;
    extern __shared__ float tile[];                         // [N][FEW_PITCH]
    int32_t *key = (int32_t *)(tile + (long)N * FEW_PITCH); // [N] the sorted rows' tokens
    uint16_t *order = (uint16_t *)(key + N);                // [N] and positions
    uint16_t *length = order + N;                           // [N] of the run that begins at a row, else 0
    // an XCD's work-groups (every eighth) take neighbouring features: rows are
    // written in pieces of 16 or 32 bytes, and only one L2 can join them to lines
    const int each = gridDim.x / 8, i0 = ((int)blockIdx.x % 8 * each + (int)blockIdx.x / 8) * FEW;
    if (i0 >= a.I)
        return;
    const int ni = min(FEW, a.I - i0), len = ni * a.B;
    // groups of four elements that cover a step's ni * B, which lie in one piece
    const int per = len / 4 + 2;
    const long groups = (long)a.T * per;
    long lo = 0, hi = 0, e = 0;
    int t = 0;
    float f[4];
    auto fetch = [&](long n) {
        t = (int)(n / per);
        lo = ((long)t * a.I + i0) * a.B;
        hi = lo + len;
        e = lo / 4 * 4 + (n - (long)t * per) * 4;
        if (e >= lo && e + 4 <= hi)
            load16(a.dX + e, f);
        else
            load_part(a.dX + e, (int)max(lo - e, 0L), (int)min(hi - e, 4L), f, 0.f);
    };
    // a thread's first group is on its way while the tokens are read
    long n = threadIdx.x;
    if (n < groups)
        fetch(n);
    const int M = q.start[a.V];
    for (int r = threadIdx.x; r < M; r += FEW_NT) {
        const int v = q.key[r];
        key[r] = v;
        order[r] = (uint16_t)q.order[r];
        length[r] = (uint16_t)(q.start[v] == r ? q.start[v + 1] - r : 0);
    }
    while (n < groups) {
        if (e < hi) {
            drop_any<4>(a.drop, e, f);
            const int r = (int)(e - lo);
            int i = r < 0 ? 0 : r / a.B, b = r - i * a.B;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (e + k >= lo && e + k < hi)
                    tile[(t * a.B + b) * FEW_PITCH + i] = f[k];
                if (++b == a.B) {
                    b = 0;
                    ++i;
                }
            }
        }
        n += FEW_NT;
        if (n < groups)
            fetch(n);
    }
    __syncthreads();
    const int i = threadIdx.x % FEW;
    if (i >= ni)
        return;
    for (int r = threadIdx.x / FEW; r < M; r += FEW_NT / FEW) {
        const int n = length[r];
        if (n == 0)
            continue;
        float sum = 0.f;
        int k = 0;
        for (; k + 8 <= n; k += 8) {
            float f[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                f[u] = tile[order[r + k + u] * FEW_PITCH + i];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                sum += f[u];
        }
        for (; k < n; ++k)
            sum += tile[order[r + k] * FEW_PITCH + i];
        put(a, a.dE + (long)key[r] * a.I + i0 + i, sum);
    }
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

Tiling tiling_of(int T, int B, int I) {
    Tiling g = {T, B, I, B, 1, (int)ceil_div(I, TILE)};
    if (B > TILE) {
        // whole eights, so that only odd batches have groups of two pieces
        g.chunks = (int)ceil_div(B, TILE);
        g.cols = (int)ceil_div(ceil_div(B, g.chunks), 8) * 8;
        g.chunks = (int)ceil_div(B, g.cols);
    }
    return g;
}

// Rows of a group of the walk: more groups while there are few rows.
int group_of(int N) { return N < 32768 ? 16 : 64; }

struct GradWs {
    int32_t *rank, *order, *key, *start;
    float *rows, *carry;
    size_t bytes;
};

// Whether a work-group can take some features of all positions.
bool few(int N, int I) { return N <= FEW_MOST && (long)N * I <= FEW_SIZE; }

GradWs layout(void *ws, int N, int I, int V) {
    char *p = (char *)ws;
    GradWs w;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char *r = p + at;
        at += align256(bytes);
        return r;
    };
    w.rank = (int32_t *)take((size_t)N * 4);
    w.order = (int32_t *)take((size_t)N * 4);
    w.key = (int32_t *)take((size_t)N * 4);
    w.start = (int32_t *)take(((size_t)V + 1) * 4);
    w.rows = (float *)take(few(N, I) ? 0 : (size_t)N * I * 4);
    w.carry = (float *)take(few(N, I) ? 0 : (size_t)ceil_div(N, group_of(N)) * 2 * I * 4);
    w.bytes = at;
    return w;
}

template <typename TS, bool PAST>
hipError_t lookup(const EmbedArgs &a, hipStream_t s) {
    const Tiling g = tiling_of(a.T, a.B, a.I);
    // runs of up to four tiles while 2048 work-groups (eight on a CU) are left
    const long steps = (long)g.T * g.chunks;
    const int run = (int)std::max(1L, std::min(4L, steps * g.tiles / 2048));
    const dim3 grid((unsigned)(steps * ceil_div(g.tiles, run)));
    if (a.B % TILE == 0 && a.drop.thr == 0)
        hipLaunchKernelGGL((embed_kernel<TS, true, false, PAST>), grid, dim3(NT), 0, s, a, g, run);
    else if (a.B % TILE == 0 && a.drop.period % 8 == 0)
        hipLaunchKernelGGL((embed_kernel<TS, true, true, PAST>), grid, dim3(NT), 0, s, a, g, run);
    else
        hipLaunchKernelGGL((embed_kernel<TS, false, true, PAST>), grid, dim3(NT), 0, s, a, g, run);
    return hipGetLastError();
}

template <int G>
hipError_t walk(const EmbedGradArgs &a, const Sorted &q, const GradWs &w, int N, hipStream_t s) {
    const int groups = (int)ceil_div(N, G);
    const int parts = (int)ceil_div(a.I, NT * 4);
    const dim3 grid((unsigned)((long)groups * parts));
    hipLaunchKernelGGL((walk_kernel<G>), grid, dim3(NT), 0, s, a, q, w.rows, w.carry, parts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || groups < 2)
        return e;
    const int cparts = (int)ceil_div(a.I, NT);
    hipLaunchKernelGGL(carry_kernel, dim3((unsigned)((long)(groups - 1) * cparts)), dim3(NT), 0, s, a, q, w.carry, G, cparts);
    return hipGetLastError();
}

} // namespace

hipError_t launch_embed(const EmbedArgs &a, bool bf16, hipStream_t s) {
    if ((long)a.T * a.I * a.B * (bf16 ? 2 : 4) >= STREAM_BYTES)
        return bf16 ? lookup<bf16_t, true>(a, s) : lookup<float, true>(a, s);
    return bf16 ? lookup<bf16_t, false>(a, s) : lookup<float, false>(a, s);
}

size_t embed_grad_ws(int T, int B, int I, int V) { return layout(nullptr, T * B, I, V).bytes; }

hipError_t launch_embed_grad(const EmbedGradArgs &a, hipStream_t s) {
    const int N = a.T * a.B;
    const GradWs w = layout(a.ws, N, a.I, a.V);
    const Sorted q = {w.rank, w.order, w.key, w.start};
    const int R = std::min(SORT_MOST, (int)ceil_div(a.V, 256));
    const long size = (long)a.V * a.I, sorters = ceil_div(a.V, R), fills = a.accumulate ? 0 : ceil_div(size, FILL);
    hipLaunchKernelGGL(sort_kernel, dim3((unsigned)(sorters + fills)), dim3(SORT_NT), 0, s, a.tokens, N, a.V, R, w.rank,
                       w.order, w.key, w.start, (int)sorters, a.dE, size);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    if (few(N, a.I)) {
        if (a.I <= 4 * FEW_CUS)
            hipLaunchKernelGGL(few_kernel<4>, dim3((unsigned)ceil_div(a.I, 32) * 8), dim3(FEW_NT), few_lds<4>(N), s, a, q, N);
        else
            hipLaunchKernelGGL(few_kernel<8>, dim3((unsigned)ceil_div(a.I, 64) * 8), dim3(FEW_NT), few_lds<8>(N), s, a, q, N);
        return hipGetLastError();
    }
    const Tiling g = tiling_of(a.T, a.B, a.I);
    // runs of up to four tiles while 2048 work-groups (eight on a CU) are left
    const long steps = (long)g.T * g.chunks;
    const int run = (int)std::max(1L, std::min(4L, steps * g.tiles / 2048));
    const dim3 grid((unsigned)(steps * ceil_div(g.tiles, run)));
    const bool whole = a.B % TILE == 0;
    if (whole && a.drop.thr == 0)
        hipLaunchKernelGGL((turn_kernel<true, false>), grid, dim3(NT), 0, s, a, g, q, w.rows, run);
    else if (whole && a.drop.period % 8 == 0)
        hipLaunchKernelGGL((turn_kernel<true, true>), grid, dim3(NT), 0, s, a, g, q, w.rows, run);
    else
        hipLaunchKernelGGL((turn_kernel<false, true>), grid, dim3(NT), 0, s, a, g, q, w.rows, run);
    if ((e = hipGetLastError()) != hipSuccess)
        return e;
    return group_of(N) == 16 ? walk<16>(a, q, w, N, s) : walk<64>(a, q, w, N, s);
}

} // namespace lstmss
