// Linear layer y = act(W x + b) + res on batch-last tensors, and its gradients.
//
//   z[t][n][b]  = sum over k of W[n][k] x[t][k][b] + bias[n],  y = act(z) + res
//   g           = dY act'(z)
//   dX[t][k][b] = sum over n of W[n][k] g[t][n][b]
//   dW[n][k]    = sum over t, b of g[t][n][b] x[t][k][b],  db[n] = the sum of g
//
// The columns of all steps are one operand of T * B rows (product.h); the
// packing launch turns each operand's contraction index innermost.
#include "head.h"
#include "product.h"

namespace lstmss {

namespace {

// ------------------------------------------------------------ packing

// A tensor whose element (o, i) is at (i / seg) * outer * seg + o * seg + i %
// seg (a matrix [outer][inner] where seg = inner; [T][outer][B] where inner = T *
// B and seg = B), times the activation's slope at z where z is given, packed with
// its inner indices as rows (`turned`), its outer ones (`straight`) or both.
struct PackJob {
    const void *p, *z;
    int inner, outer, seg, act;
    bool bf16, z_bf16;
    int planes, ks_turned, ks_straight;
    uint4 *turned, *straight;
    float *sums; // [ceil(inner / 64)][outer]: sums over 64 inner indices, or NULL
    int first;   // work-group
};

struct PackJobs {
    PackJob job[4];
    int n;
};

// 16 values of a thread from memory to the tile in LDS, W neighbours at a time.
template <int W, bool BF16, bool Z>
__device__ __forceinline__ void pack_fetch(const PackJob &j, int o0, int i0, float *tile) {
    constexpr int LANES = 64 / W, STEP = 256 / LANES; // threads along 64 inner indices; outer ones at a time
    const int i = i0 + threadIdx.x % LANES * W, o = threadIdx.x / LANES, q = i / j.seg;
    const bool there = i < j.inner;
    const long at = (long)q * j.outer * j.seg + (i - q * j.seg);
    float v[64 / STEP][W];
#pragma unroll
    for (int r = 0; r < 64 / STEP; ++r) {
        const int row = o0 + o + r * STEP;
        if (there && row < j.outer) {
            const long a = at + (long)row * j.seg;
            if constexpr (W == 1)
                v[r][0] = load_any(j.p, a, j.bf16);
            else if constexpr (BF16)
                load16((const bf16_t *)j.p + a, v[r]);
            else
                load16((const float *)j.p + a, v[r]);
        } else {
#pragma unroll
            for (int e = 0; e < W; ++e)
                v[r][e] = 0.f;
        }
    }
    if (Z) {
#pragma unroll
        for (int r = 0; r < 64 / STEP; ++r) {
            const int row = o0 + o + r * STEP;
            if (there && row < j.outer) {
                const long a = at + (long)row * j.seg;
#pragma unroll
                for (int e = 0; e < W; ++e)
                    v[r][e] *= act_slope(load_any(j.z, a + e, j.z_bf16), j.act);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 64 / STEP; ++r) {
        float *to = tile + (o + r * STEP) * 68 + (i - i0);
        if constexpr (W == 1) {
            to[0] = v[r][0];
        } else {
#pragma unroll
            for (int e = 0; e < W; e += 4)
                *(f32x4 *)(to + e) = *(f32x4 *)(v[r] + e);
        }
    }
}

// A work-group: 64 x 64 values through LDS (rows of 68 floats: 16-byte reads down
// 16 rows fall on all banks), read from memory once, in runs, and stored as
// whole blocks, a wavefront's 1 KB at once.  Memory bound: 5.0 to 5.6 TB/s on
// large tensors.
__global__ void __launch_bounds__(256) pack_kernel(const PackJobs jobs) {
    __shared__ float tile[64 * 68];
    __shared__ float part[4][64];
    int n = 0;
    while (n + 1 < jobs.n && (int)blockIdx.x >= jobs.job[n + 1].first)
        ++n;
    const PackJob &j = jobs.job[n];
    const int across = (j.inner + 63) / 64;
    const int id = blockIdx.x - j.first, to = id / across, ti = id - to * across;
    const int o0 = to * 64, i0 = ti * 64, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (j.z) {
        if (j.bf16 && j.seg % 8 == 0)
            pack_fetch<8, true, true>(j, o0, i0, tile);
        else if (!j.bf16 && j.seg % 4 == 0)
            pack_fetch<4, false, true>(j, o0, i0, tile);
        else
            pack_fetch<1, false, true>(j, o0, i0, tile);
    } else {
        if (j.bf16 && j.seg % 8 == 0)
            pack_fetch<8, true, false>(j, o0, i0, tile);
        else if (!j.bf16 && j.seg % 4 == 0)
            pack_fetch<4, false, false>(j, o0, i0, tile);
        else
            pack_fetch<1, false, false>(j, o0, i0, tile);
    }
    __syncthreads();
    float v[8];
    if (j.turned)
#pragma unroll
        for (int r = 0; r < 2; ++r) { // blocks of rows; a wavefront has one of the four of k
            const float *from = tile + (w * 16 + (lane >> 5) * 8) * 68 + r * 32 + (lane & 31);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = from[e * 68];
            if (i0 + r * 32 < j.inner)
                pack_piece(j.turned + ((long)(ti * 2 + r) * j.ks_turned + to * 4 + w) * j.planes * 64, lane, j.planes, v);
        }
    if (!j.straight && !j.sums)
        return;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const f32x4 *from = (const f32x4 *)(tile + (r * 32 + (lane & 31)) * 68 + w * 16 + (lane >> 5) * 8);
        *(f32x4 *)v = from[0];
        *(f32x4 *)(v + 4) = from[1];
        if (j.straight && o0 + r * 32 < j.outer)
            pack_piece(j.straight + ((long)(to * 2 + r) * j.ks_straight + ti * 4 + w) * j.planes * 64, lane, j.planes, v);
        if (j.sums) {
            float sum = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
            sum += __shfl_xor(sum, 32, 64);
            if (lane < 32)
                part[w][r * 32 + lane] = sum;
        }
    }
    if (j.sums) {
        __syncthreads();
        const int o = threadIdx.x;
        if (o < 64 && o0 + o < j.outer)
            j.sums[(long)ti * j.outer + o0 + o] = (part[0][o] + part[1][o]) + (part[2][o] + part[3][o]);
    }
}

// db from the chunks' sums: 8 threads of a column take every eighth, and are added
// up in their order.
__global__ void __launch_bounds__(256) bias_grad_kernel(int N, int chunks, const float *sums, bool accumulate,
                                                        float *db) {
    __shared__ float part[8][32];
    const int c = threadIdx.x & 31, q = threadIdx.x >> 5, n = blockIdx.x * 32 + c;
    if (n < N)
        part[q][c] = sum_parts<16>(0.f, sums + (long)q * N + n, (chunks - q + 7) / 8, 8l * N);
    __syncthreads();
    if (q == 0 && n < N) {
        float s = accumulate ? db[n] : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            s += part[i][c];
        db[n] = s;
    }
}

// ------------------------------------------------------------ epilogues

// y [T][N][B] (and z) at rows n, columns (t, b).  Where WIDE divides the batch
// WIDE columns are neighbours in memory.
template <typename TS>
struct Forward {
    static constexpr int WIDE = vec_of<TS>();
    int N, B, J, act;
    const float *b;
    const TS *res;
    TS *y, *z;
    struct Ahead {
        float bias, res[WIDE];
    };
    __device__ __forceinline__ Ahead ahead(int, int row, int col) const {
        Ahead a;
        a.bias = b ? b[row] : -0.f; // (-0 + v is v, whatever its sign)
#pragma unroll
        for (int e = 0; e < WIDE; ++e)
            a.res[e] = -0.f;
        if (!res)
            return a;
        int t = col / B, at = col - t * B;
        long i = ((long)t * N + row) * B + at;
        if (B % WIDE == 0) {
            load16(res + i, a.res);
        } else {
#pragma unroll
            for (int e = 0; e < WIDE; ++e) {
                if (col + e < J)
                    a.res[e] = st<TS>::load(res, i);
                ++i;
                if (++at == B) {
                    at = 0;
                    i += (long)(N - 1) * B;
                }
            }
        }
        return a;
    }
    __device__ __forceinline__ void span(int, int row, int col, const float *v, const Ahead &a) const {
        int t = col / B, at = col - t * B;
        long i = ((long)t * N + row) * B + at;
        float s[WIDE], o[WIDE];
#pragma unroll
        for (int e = 0; e < WIDE; ++e)
            s[e] = v[e] + a.bias;
#pragma unroll
        for (int e = 0; e < WIDE; ++e)
            o[e] = act_value(s[e], act) + a.res[e];
        if (B % WIDE == 0) {
            if (z)
                store16(z + i, s);
            store16(y + i, o);
            return;
        }
#pragma unroll
        for (int e = 0; e < WIDE; ++e) {
            if (col + e >= J)
                return;
            if (z)
                st<TS>::store(z, i, s[e]);
            st<TS>::store(y, i, o[e]);
            ++i;
            if (++at == B) {
                at = 0;
                i += (long)(N - 1) * B;
            }
        }
    }
    __device__ __forceinline__ void one(int row, int col, float v) const {
        const int t = col / B;
        const long i = ((long)t * N + row) * B + (col - t * B);
        if (b)
            v += b[row];
        if (z)
            st<TS>::store(z, i, v);
        const float o = act_value(v, act);
        st<TS>::store(y, i, res ? o + st<TS>::load(res, i) : o);
    }
};

// dX [T][K][B] at rows k, columns (t, b).
struct InputGrad {
    static constexpr int WIDE = 4;
    int K, B, J;
    float *dX;
    typedef Nothing Ahead;
    __device__ __forceinline__ Nothing ahead(int, int, int) const { return {}; }
    __device__ __forceinline__ void span(int, int row, int col, const float *v, Nothing) const {
        int t = col / B, at = col - t * B;
        long i = ((long)t * K + row) * B + at;
        if (B % WIDE == 0) {
            store16(dX + i, v);
            return;
        }
#pragma unroll
        for (int e = 0; e < WIDE; ++e) {
            if (col + e >= J)
                return;
            dX[i++] = v[e];
            if (++at == B) {
                at = 0;
                i += (long)(K - 1) * B;
            }
        }
    }
};

// dW [N][K] at rows n, columns k.
struct WeightGrad {
    static constexpr int WIDE = 4;
    int N, K;
    bool accumulate;
    float *dW;
    struct Ahead {
        float old[WIDE];
    };
    __device__ __forceinline__ Ahead ahead(int, int row, int col) const {
        Ahead a;
        const float *p = dW + (long)row * K + col;
        if (accumulate && K - col >= WIDE)
            load16(p, a.old);
        else
            load_part(p, 0, accumulate ? K - col : 0, a.old, 0.f);
        return a;
    }
    __device__ __forceinline__ void span(int, int row, int col, const float *v, const Ahead &a) const {
        float o[WIDE];
#pragma unroll
        for (int e = 0; e < WIDE; ++e)
            o[e] = a.old[e] + v[e];
        store_row(dW + (long)row * K + col, K - col, o);
    }
};

// ------------------------------------------------------------ plans

constexpr int K_UNIT = 4; // blocks of k are padded to whole stages of any tile

int ks_of(long k) { return (int)(ceil_div(k, 16 * K_UNIT) * K_UNIT); }
size_t packed_bytes(long rows, long k, int planes) { return (size_t)ceil_div(rows, 32) * ks_of(k) * planes * 1024; }

// Tiles of a product; the tiles from `whole` on are cut into `splits`.
enum Tile { TILE_256, TILE_256x128, TILE_128, TILE_64, TILES };
struct Plan {
    Tile tile;
    int whole, splits, split_ks;
};

// What a tile takes for a block of 16 k, in us, alone on its CU and where CUs have
// several, and how much of its epilogue's time at a CU's share of memory is seen:
// fitted to every tile and cut, measured on 31 products of 517 to 32000 rows, 640 to
// 25600 columns and 494 to 4096 k, with and without z and residual.  Against all cuts
// into 2 to 16, timed with operands in memory, the choice is within 1 % of the quickest
// for 26 of the 32 fp32 calls and within 8 % for all (0.8 % in the mean), for 21 of the
// 30 in bf16 within 1 %, for 27 within 8 % and for all within 11 %.
struct TileCost {
    int rows, columns;
    float alone, shared; // us
    float ends;
};
constexpr TileCost COST_1[TILES] = {{256, 256, 0.33f, 0.45f, 1.25f},
                                    {256, 128, 0.25f, 0.23f, 1.f},
                                    {128, 128, 0.155f, 0.125f, 1.f},
                                    {64, 64, 0.055f, 0.052f, 0.75f}};
constexpr TileCost COST_6[TILES] = {{}, {}, {128, 128, 0.64f, 0.47f, 1.f}, {64, 64, 0.26f, 0.165f, 0.75f}};

// The least of estimated times of an M x N product over KS blocks of k in
// `products` matrix instructions, whose epilogue moves `out` bytes an element (a
// layer's: y, z and the residual, whether they are there or not).  All sums are cut,
// or those of the tiles that are over whole rounds of the CUs (128 x 128 fp32 tiles,
// 800 of 128 blocks of k: 322 -> 285 us).
Plan plan_product(long M, long N, int KS, int products, int out) {
    Plan best = {};
    double least = 1e300;
    const float scale = products == 3 ? 0.55f : 1.f; // (three products: half the instructions of six)
    for (int t = products == 1 ? TILE_256 : TILE_128; t < TILES; ++t) {
        const TileCost &c = products == 1 ? COST_1[t] : COST_6[t];
        const long tiles = ceil_div(M, c.rows) * ceil_div(N, c.columns);
        // us of `count` sums over `ks` blocks of k, and of `bytes` an element after each
        auto side_by_side = [&](long count, int ks, int bytes) {
            const long rounds = ceil_div(count, 256); // of the busiest CU
            return rounds * (ks * (double)(rounds > 1 ? c.shared : c.alone) * scale +
                             c.ends * (c.rows * c.columns * bytes / 18.75e3));
        };
        for (int part = 0; part < 2; ++part) { // all tiles, or those over whole rounds
            const long rest = part == 0 ? tiles : tiles % 256, whole = tiles - rest;
            if (part == 1 && (rest == 0 || whole == 0))
                continue;
            for (int splits = part == 0 ? 1 : 2; splits <= 16; ++splits) {
                const int each = (int)(ceil_div(ceil_div(KS, splits), K_UNIT) * K_UNIT);
                if (splits > 1 && (each < 2 * K_UNIT || (long)each * (splits - 1) >= KS))
                    continue;
                double us = 5.0 + side_by_side(rest * splits, each, splits > 1 ? 4 : out);
                if (whole > 0)
                    us += side_by_side(whole, KS, out);
                if (splits > 1)
                    us += 3.5 + (double)rest * c.rows * c.columns * (splits / 2.5e6 + out / 4.0e6);
                if (us < least) {
                    least = us;
                    best = {(Tile)t, (int)(splits > 1 ? whole : tiles), splits, each};
                }
            }
        }
    }
    return best;
}

size_t part_bytes(const Plan &p, long M, long N) {
    const size_t rows = COST_1[p.tile].rows, columns = COST_1[p.tile].columns;
    return p.splits > 1 ? (ceil_div(M, rows) * ceil_div(N, columns) - p.whole) * p.splits * rows * columns * 4 : 0;
}

template <int PA, int PB, class Epi>
hipError_t run_product(Product g, const Plan &p, const Epi &epi, hipStream_t s) {
    g.tm = (int)ceil_div(g.M, COST_1[p.tile].rows);
    g.tn = (int)ceil_div(g.N, COST_1[p.tile].columns);
    g.tiles = g.tm * g.tn;
    g.batch = 1;
    g.whole = p.whole;
    g.splits = p.splits;
    g.split_ks = p.split_ks;
    g.symmetric = false;
    const int rest = g.tiles - g.whole, groups = g.whole + rest * g.splits;
    const dim3 grid((unsigned)groups);
    // The small partial products of three planes have sums of their own (TWO): cut
    // off below a large sum towards minus infinity they leave a mean, -8e-7 of the
    // result's size after 32000 terms, where this has none (and errors of 2.7e-7
    // for 7e-7 after 8192).  256 rows or columns leave no registers for that; they
    // took 250 TFLOP/s where 128 take 235 on sizes that suit both.
    if constexpr (PA * PB == 1) {
        switch (p.tile) {
        case TILE_256: product_kernel<1, 1, 4, 2, 2, 4, 4, 2, false, true, 1><<<grid, 512, 0, s>>>(g, epi); break;
        case TILE_256x128: product_kernel<1, 1, 4, 2, 2, 2, 2, 3, false, true, 2><<<grid, 256, 0, s>>>(g, epi); break;
        case TILE_128: product_kernel<1, 1, 2, 2, 2, 2, 4, 2, false, true, 2><<<grid, 256, 0, s>>>(g, epi); break;
        default: product_kernel<1, 1, 1, 1, 2, 2, 4, 3, false, false, 2><<<grid, 256, 0, s>>>(g, epi);
        }
    } else {
        // (64 x 64: three stages for one or two work-groups to a CU, 23.8 us for 26.3
        // with two on 231 tiles of 82 blocks of k; two stages for three, 704 us for 743 on 4096)
        if (p.tile == TILE_128)
            product_kernel<PA, PB, 2, 2, 2, 2, 1, 3, true, false, 2><<<grid, 256, 0, s>>>(g, epi);
        else if (groups <= 512)
            product_kernel<PA, PB, 1, 1, 2, 2, 2, 3, true, true, 2><<<grid, 256, 0, s>>>(g, epi);
        else
            product_kernel<PA, PB, 1, 1, 2, 2, 2, 2, true, false, 3><<<grid, 256, 0, s>>>(g, epi);
    }
    if (rest > 0) {
        const int bm = COST_1[p.tile].rows, bn = COST_1[p.tile].columns;
        const long threads = (long)rest * bm * (bn / Epi::WIDE);
        product_join_kernel<<<dim3((unsigned)ceil_div(threads, 256)), 256, 0, s>>>(g, bm, bn, epi);
    }
    return hipGetLastError();
}

Source source(const void *p, bool bf16, long rows, long ks, int seg, bool inner_k) {
    Source s = {};
    s.p = p;
    s.bf16 = bf16;
    s.rows = (int)rows;
    s.ks = (int)ks;
    s.seg = seg;
    s.inner_k = inner_k;
    return s;
}

struct Packer {
    PackJobs jobs = {};
    int groups = 0;
    // `s` packed into `out`, and, where `other` is given, its transpose there.
    const uint4 *add(const Source &s, int planes, uint4 *out, uint4 *other = nullptr, float *sums = nullptr) {
        PackJob &j = jobs.job[jobs.n++];
        j.p = s.p;
        j.z = s.z;
        j.inner = s.inner_k ? s.ks : s.rows;
        j.outer = s.inner_k ? s.rows : s.ks;
        j.seg = s.seg;
        j.act = s.act;
        j.bf16 = s.bf16;
        j.z_bf16 = s.z_bf16;
        j.planes = planes;
        j.ks_turned = ks_of(j.outer);
        j.ks_straight = ks_of(j.inner);
        j.turned = s.inner_k ? other : out;
        j.straight = s.inner_k ? out : other;
        j.sums = sums;
        j.first = groups;
        groups += (int)(ceil_div(j.inner, 64) * ceil_div(j.outer, 64));
        return out;
    }
    hipError_t run(hipStream_t s) {
        pack_kernel<<<dim3((unsigned)groups), 256, 0, s>>>(jobs);
        return hipGetLastError();
    }
};

// Consecutive places in the workspace.
struct Space {
    char *at;
    template <typename T>
    T *take(size_t bytes) {
        T *p = (T *)at;
        at += (bytes + 255) / 256 * 256;
        return p;
    }
};

float unscale_of(int pa, int pb) { return (pa == 3 ? 0x1p-24f : 1.f) * (pb == 3 ? 0x1p-24f : 1.f); }

// ------------------------------------------------------------ few columns

// Few columns (a step of a server's sequences or beams): W is read once for 32 of
// them, from where it is, and nothing is packed.
//
// A work-group goes over tiles of 16 rows, its WK wavefronts share the
// contraction; a wavefront keeps its part of x in registers for all tiles (the
// matrix instruction's second operand: column lane % 16, and the four groups of
// 16 lanes take consecutive 16 bytes of k), so that what streams is W alone, 64
// bytes of each of 16 rows an instruction, the rows of as many tiles (DEPTH) on their
// way as the registers hold.  fp32 is multiplied by the fp32 instructions (memory
// sets the time), one for each of the four k that 16 bytes hold.  W of 32000 x
// 4096 in bf16, 16 columns: 47 us, 5.6 TB/s.

// Where this is the quicker way (us, this way / packed): 64 columns, 32000 x 4096
// bf16 108 / 149 and fp32 280 / 412, 10000 x 650 fp32 21 / 28; 128 columns, 32000 x
// 4096 bf16 194 / 162, 10000 x 650 fp32 36 / 31, 2048 x 2048 fp32 22 / 23, 512 x 512
// bf16 4.2 / 9.8.
bool few_columns(long J, int K, int N) {
    return K >= 8 && (J <= 64 || (J <= 128 && (long)N * K <= 1l << 22));
}

// 16-byte loads of W of a lane and tile, for NT times 16 columns: what 128
// registers (four wavefronts a SIMD) hold beside x.
constexpr int few_units(int NT) { return NT == 1 ? 8 : 4; }

template <typename TS>
constexpr int few_k() { // k of a unit
    return 4 * vec_of<TS>();
}

template <typename TS>
struct Few {
    int N, K, J, B;
    int tiles, units; // of a wavefront
    int chunk;        // k of a work-group
    const TS *W, *x;
    float *part; // [gridDim.y][N][J] where the contraction is cut
};

// The elements of 16 bytes from number `from` on, the others zero.
template <typename TS>
__device__ __forceinline__ u32x4 keep_from(u32x4 v, int from) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        if constexpr (vec_of<TS>() == 4)
            v[d] = d >= from ? v[d] : 0u;
        else
            v[d] = 2 * d >= from ? v[d] : 2 * d + 1 >= from ? v[d] & 0xffff0000u : 0u;
    }
    return v;
}

// No load is under a condition but a wavefront's: rows, columns and k past the end
// are read as the last ones, and what is read twice so is zero.  (8192 x 2048
// bf16, one column: 14.3 us with a branch for each lane's loads, 20 KB of code, and
// 9.7 us so.)
template <typename TS, int NT, int WK, int UNITS, int DEPTH, class Epi>
__global__ void __launch_bounds__(64 * WK, 4) linear_few_kernel(const Few<TS> a, const Epi epi) {
    constexpr int VEC = vec_of<TS>(), UK = few_k<TS>();
    __shared__ f32x4 part[2][WK][NT][64];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = blockIdx.y * a.chunk + w * a.units * UK, group = (lane >> 4) * VEC;
    const int kend = min(a.K, (int)(blockIdx.y + 1) * a.chunk);
    const int col0 = blockIdx.z * NT * 16;
    u32x4 ahead[DEPTH][UNITS];
    auto fetch = [&](u32x4 (&rows)[UNITS], int tile) __attribute__((always_inline)) {
        const TS *p = a.W + (long)min(tile * 16 + (lane & 15), a.N - 1) * a.K;
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
            if (u < a.units) {
                const int k = first + u * UK + group, at = min(k, kend - VEC);
                rows[u] = *(const typename vec<TS>::raw *)(p + at);
                if (first + (u + 1) * UK > kend)
                    rows[u] = keep_from<TS>(rows[u], k - at);
            }
    };
    const int step = gridDim.x;
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (d == 0 || (int)blockIdx.x + d * step < a.tiles)
            fetch(ahead[d], blockIdx.x + d * step);
    u32x4 xs[NT][UNITS];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int col = min(col0 + j * 16 + (lane & 15), a.J - 1), t = col / a.B;
        const TS *p = a.x + (long)t * a.K * a.B + (col - t * a.B);
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
            if (u < a.units) {
                const int k = first + u * UK + group, at = min(k, kend - VEC);
                const TS *q = p + (long)at * a.B;
                if constexpr (VEC == 4) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        xs[j][u][e] = __float_as_uint(q[(long)e * a.B]);
                } else {
#pragma unroll
                    for (int d = 0; d < 4; ++d)
                        xs[j][u][d] = q[(long)(2 * d) * a.B].bits | (uint32_t)q[(long)(2 * d + 1) * a.B].bits << 16;
                }
                if (first + (u + 1) * UK > kend)
                    xs[j][u] = keep_from<TS>(xs[j][u], k - at);
            }
    }
    auto one = [&](u32x4 (&rows)[UNITS], int it, int tile) __attribute__((always_inline)) {
        f32x4 acc[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j)
            acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
            if (u < a.units) {
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    if constexpr (VEC == 8) {
                        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, rows[u]),
                                                                         __builtin_bit_cast(bf16x8, xs[j][u]), acc[j],
                                                                         0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(rows[u][e]),
                                                                          __uint_as_float(xs[j][u][e]), acc[j], 0, 0, 0);
                    }
                }
            }
        if (tile + DEPTH * step < a.tiles)
            fetch(rows, tile + DEPTH * step);
#pragma unroll
        for (int j = 0; j < NT; ++j)
            part[it & 1][w][j][lane] = acc[j];
        lds_barrier(); // (the buffer before this one is read by then: one barrier a tile)
        // a wavefront adds up every fourth row of 16 columns
#pragma unroll 1
        for (int q = w; q < 4 * NT; q += WK) {
            const int j = q >> 2, e = q & 3;
            const float *from = (const float *)&part[it & 1][0][j][lane] + e;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < WK; ++i)
                sum += from[i * NT * 256];
            const int row = tile * 16 + 4 * (lane >> 4) + e, col = col0 + j * 16 + (lane & 15);
            if (row < a.N && col < a.J) {
                if (gridDim.y > 1)
                    a.part[((long)blockIdx.y * a.N + row) * a.J + col] = sum;
                else
                    epi.one(row, col, sum);
            }
        }
    };
    int it = 0;
    for (int tile = blockIdx.x; tile < a.tiles; tile += DEPTH * step)
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (d == 0 || tile + d * step < a.tiles)
                one(ahead[d], it++, tile + d * step);
}

// Sums of the cuts, in their order, and the epilogue: a thread has a row and column.
template <class Epi>
__global__ void __launch_bounds__(256) few_join_kernel(int N, int J, int cuts, const float *part, const Epi epi) {
    const int at = blockIdx.x * 256 + threadIdx.x, row = at / J;
    if (row < N)
        epi.one(row, at - row * J, sum_parts<4>(0.f, part + at, cuts, (long)N * J));
}

// How the contraction of K is cut: work-groups, and wavefronts of one.
struct FewPlan {
    int cuts, waves, units;
};

// Wavefronts of a work-group: two or more units each, at most 16 (K = 650 in fp32,
// 10000 rows: 16 of 3 units 10.4 us, 8 of 6 11.8 us).
FewPlan plan_few(int K, int unit_k, int most) {
    FewPlan p;
    const int units = (int)ceil_div(K, unit_k);
    p.cuts = (int)ceil_div(units, 16 * most);
    const int each = (int)ceil_div(units, p.cuts);
    p.waves = 1;
    while (p.waves < 16 && p.waves * 4 <= each)
        p.waves *= 2;
    p.units = (int)ceil_div(each, p.waves);
    return p;
}

// Tiles of a work-group: so that the busiest CU has the fewest, and of those
// numbers the largest, whose x is read least often.
int tiles_each(int tiles, int beside) {
    int best = 1;
    long least = 1l << 60;
    for (int per = 1; per <= 64; ++per) {
        const long busy = ceil_div(ceil_div(tiles, per) * beside, 256) * per;
        if (busy <= least) {
            least = busy;
            best = per;
        }
    }
    return best;
}

size_t few_ws(long J, int K, int N, bool bf16) {
    const FewPlan p = plan_few(K, bf16 ? few_k<bf16_t>() : few_k<float>(), few_units(J <= 16 ? 1 : 2));
    return p.cuts > 1 ? (size_t)p.cuts * N * J * 4 : 0;
}

template <typename TS, int NT, int UNITS, int DEPTH, class Epi>
void few_waves(int waves, dim3 grid, const Few<TS> &f, const Epi &epi, hipStream_t s) {
    switch (waves) {
    case 1: linear_few_kernel<TS, NT, 1, UNITS, DEPTH><<<grid, 64, 0, s>>>(f, epi); break;
    case 2: linear_few_kernel<TS, NT, 2, UNITS, DEPTH><<<grid, 128, 0, s>>>(f, epi); break;
    case 4: linear_few_kernel<TS, NT, 4, UNITS, DEPTH><<<grid, 256, 0, s>>>(f, epi); break;
    case 8: linear_few_kernel<TS, NT, 8, UNITS, DEPTH><<<grid, 512, 0, s>>>(f, epi); break;
    default: linear_few_kernel<TS, NT, 16, UNITS, DEPTH><<<grid, 1024, 0, s>>>(f, epi); break;
    }
}

template <typename TS, int NT, class Epi>
hipError_t run_few(const LinearArgs &a, const Epi &epi, hipStream_t s) {
    const FewPlan p = plan_few(a.K, few_k<TS>(), few_units(NT));
    Few<TS> f;
    f.N = a.N;
    f.K = a.K;
    f.J = a.T * a.B;
    f.B = a.B;
    f.tiles = (int)ceil_div(a.N, 16);
    f.units = p.units;
    f.chunk = p.units * p.waves * few_k<TS>();
    f.W = (const TS *)a.W;
    f.x = (const TS *)a.x;
    f.part = (float *)a.ws;
    const int per = tiles_each(f.tiles, p.cuts * (int)ceil_div(f.J, NT * 16));
    const dim3 grid((unsigned)ceil_div(f.tiles, per), (unsigned)p.cuts, (unsigned)ceil_div(f.J, NT * 16));
    // tiles on their way (one / these, us, W from memory: 10000 x 650 fp32 14.2 / 13.0;
    // 30000 x 1024 bf16 22.8 / 19.4; 512 x 512 bf16 3.9 / 2.9)
    constexpr int most = few_units(NT);
    if (p.units <= most / 4)
        few_waves<TS, NT, most / 4, 4>(p.waves, grid, f, epi, s);
    else if (p.units <= most / 2)
        few_waves<TS, NT, most / 2, NT == 1 ? 3 : 2>(p.waves, grid, f, epi, s);
    else
        few_waves<TS, NT, most, 1>(p.waves, grid, f, epi, s);
    if (p.cuts > 1)
        few_join_kernel<<<dim3((unsigned)ceil_div((long)a.N * f.J, 256)), 256, 0, s>>>(a.N, f.J, p.cuts, f.part, epi);
    return hipGetLastError();
}

template <typename TS>
hipError_t linear_typed(const LinearArgs &a, hipStream_t s) {
    constexpr int P = sizeof(TS) == 4 ? 3 : 1;
    const long J = (long)a.T * a.B;
    Forward<TS> epi;
    epi.N = a.N;
    epi.B = a.B;
    epi.J = (int)J;
    epi.act = a.act;
    epi.b = a.b;
    epi.res = (const TS *)a.res;
    epi.y = (TS *)a.y;
    epi.z = (TS *)a.z;
    if (few_columns(J, a.K, a.N))
        return J <= 16 ? run_few<TS, 1>(a, epi, s) : run_few<TS, 2>(a, epi, s);
    const Plan p = plan_product(a.N, J, ks_of(a.K), P == 3 ? 6 : 1, 3 * (int)sizeof(TS));
    Space sp = {(char *)a.ws};
    Packer pk;
    Product g = {};
    g.sa = source(a.W, a.bf16, a.N, a.K, a.K, true);
    g.sb = source(a.x, a.bf16, J, a.K, a.B, false);
    g.sources = P == 3;
    g.A = pk.add(g.sa, P, sp.take<uint4>(packed_bytes(a.N, a.K, P)));
    g.B = pk.add(g.sb, P, sp.take<uint4>(packed_bytes(J, a.K, P)));
    g.part = sp.take<float>(part_bytes(p, a.N, J));
    g.M = a.N;
    g.N = (int)J;
    g.KS = ks_of(a.K);
    g.unscale = unscale_of(P, P);
    if (hipError_t e = pk.run(s))
        return e;
    return run_product<P, P>(g, p, epi, s);
}

template <int PW, int PG>
hipError_t grad_typed(const LinearGradArgs &a, hipStream_t s) {
    constexpr int PX = PW; // x and W are of one type
    constexpr int PRODUCTS = PW * PG == 9 ? 6 : PW * PG;
    const long J = (long)a.T * a.B;
    const Plan px = plan_product(a.K, J, ks_of(a.N), PRODUCTS, 4), pw = plan_product(a.N, a.K, ks_of(J), PRODUCTS, 4);
    Space sp = {(char *)a.ws};
    Packer pk;
    auto with_z = [&](Source q) {
        q.z = a.act == ACT_NONE ? nullptr : a.z;
        q.act = a.act;
        q.z_bf16 = a.bf16;
        return q;
    };
    Product gx = {}, gw = {};
    const int chunks = (int)ceil_div(J, 64);
    uint4 *columns = a.dX ? sp.take<uint4>(packed_bytes(J, a.N, PG)) : nullptr;
    uint4 *rows = a.dW ? sp.take<uint4>(packed_bytes(a.N, J, PG)) : nullptr;
    float *sums = a.db ? sp.take<float>((size_t)chunks * a.N * 4) : nullptr;
    gx.sa = source(a.W, a.bf16, a.K, a.N, a.K, false);
    gx.sb = with_z(source(a.dY, a.dy_bf16, J, a.N, a.B, false));
    gw.sa = with_z(source(a.dY, a.dy_bf16, a.N, J, a.B, true));
    gw.sb = source(a.x, a.bf16, a.K, J, a.B, true);
    pk.add(gx.sb, PG, columns, rows, sums); // g is read once for both products and for db
    if (a.dX) {
        gx.A = pk.add(gx.sa, PW, sp.take<uint4>(packed_bytes(a.K, a.N, PW)));
        gx.B = columns;
        gx.part = sp.take<float>(part_bytes(px, a.K, J));
        gx.M = a.K;
        gx.N = (int)J;
        gx.KS = ks_of(a.N);
        gx.unscale = unscale_of(PW, PG);
        gx.sources = PRODUCTS > 1;
    }
    if (a.dW) {
        gw.A = rows;
        gw.B = pk.add(gw.sb, PX, sp.take<uint4>(packed_bytes(a.K, J, PX)));
        gw.part = sp.take<float>(part_bytes(pw, a.N, a.K));
        gw.M = a.N;
        gw.N = a.K;
        gw.KS = ks_of(J);
        gw.unscale = unscale_of(PG, PX);
        gw.sources = PRODUCTS > 1;
    }
    if (hipError_t e = pk.run(s))
        return e;
    if (a.dX) {
        InputGrad epi;
        epi.K = a.K;
        epi.B = a.B;
        epi.J = (int)J;
        epi.dX = a.dX;
        if (hipError_t e = run_product<PW, PG>(gx, px, epi, s))
            return e;
    }
    if (a.dW) {
        WeightGrad epi;
        epi.N = a.N;
        epi.K = a.K;
        epi.accumulate = a.accumulate;
        epi.dW = a.dW;
        if (hipError_t e = run_product<PG, PX>(gw, pw, epi, s))
            return e;
    }
    if (a.db)
        bias_grad_kernel<<<dim3((unsigned)ceil_div(a.N, 32)), 256, 0, s>>>(a.N, chunks, sums, a.accumulate, a.db);
    return hipGetLastError();
}

// Planes of g: what is of bf16 and not multiplied by a slope is whole in one.
int grad_planes(bool bf16, bool dy_bf16, int act) { return bf16 && dy_bf16 && act == ACT_NONE ? 1 : 3; }

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

} // namespace

size_t linear_ws(int T, int B, int K, int N, bool bf16) {
    const int P = bf16 ? 1 : 3;
    const long J = (long)T * B;
    if (few_columns(J, K, N))
        return few_ws(J, K, N, bf16);
    const Plan p = plan_product(N, J, ks_of(K), P == 3 ? 6 : 1, bf16 ? 6 : 12);
    return round256(packed_bytes(N, K, P)) + round256(packed_bytes(J, K, P)) + round256(part_bytes(p, N, J));
}

hipError_t launch_linear(const LinearArgs &a, hipStream_t s) {
    return a.bf16 ? linear_typed<bf16_t>(a, s) : linear_typed<float>(a, s);
}

size_t linear_grad_ws(int T, int B, int K, int N, bool bf16, bool dy_bf16, int act) {
    const int P = bf16 ? 1 : 3, PG = grad_planes(bf16, dy_bf16, act), products = P * PG == 9 ? 6 : P * PG;
    const long J = (long)T * B;
    const Plan px = plan_product(K, J, ks_of(N), products, 4), pw = plan_product(N, K, ks_of(J), products, 4);
    return round256(packed_bytes(K, N, P)) + round256(packed_bytes(J, N, PG)) + round256(part_bytes(px, K, J)) +
           round256((size_t)ceil_div(J, 64) * N * 4) + round256(packed_bytes(N, J, PG)) +
           round256(packed_bytes(K, J, P)) + round256(part_bytes(pw, N, K));
}

hipError_t launch_linear_grad(const LinearGradArgs &a, hipStream_t s) {
    const int pg = grad_planes(a.bf16, a.dy_bf16, a.act);
    if (!a.bf16)
        return grad_typed<3, 3>(a, s);
    return pg == 1 ? grad_typed<1, 1>(a, s) : grad_typed<1, 3>(a, s);
}

} // namespace lstmss
