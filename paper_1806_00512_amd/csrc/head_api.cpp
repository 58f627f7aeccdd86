// Host side of the operators of a language model's head: argument checks and
// launches, in one translation unit with the entry points below them.
#include "language_api.cpp"

#include "head.h"

#include <initializer_list>

namespace {

// Memory of an argument (at NULL: none).
struct Span {
    const void *at;
    int64_t bytes;
};

// Outputs that share memory with an input or with another output.
bool meets(std::initializer_list<Span> outputs, std::initializer_list<Span> inputs) {
    auto shared = [](const Span &a, const Span &b) {
        const uintptr_t p = (uintptr_t)a.at, q = (uintptr_t)b.at;
        return p && q && a.bytes > 0 && b.bytes > 0 && (p < q ? q - p < (uintptr_t)a.bytes : p - q < (uintptr_t)b.bytes);
    };
    for (auto o = outputs.begin(); o != outputs.end(); ++o) {
        for (const Span &i : inputs)
            if (shared(*o, i))
                return true;
        for (auto p = outputs.begin(); p != o; ++p)
            if (shared(*o, *p))
                return true;
    }
    return false;
}

// An input that may be the output `out` itself, but not share a part of it.
Span or_out(const void *in, const void *out, int64_t bytes) { return {in == out ? nullptr : in, bytes}; }

int64_t size_of(int32_t dtype) { return dtype == LSTMSS_BF16 ? 2 : 4; }

int32_t check_linear(const lstmss_linear_dims *d) {
    if (!d)
        return fail(LSTMSS_ERR_INVALID_ARG, "sizes are NULL");
    if (d->T < 1 || d->B < 1 || d->K < 1 || d->N < 1)
        return fail(LSTMSS_ERR_INVALID_ARG, "sizes must be positive (T=%d B=%d K=%d N=%d)", d->T, d->B,
                    d->K, d->N);
    if (d->dtype != LSTMSS_F32 && d->dtype != LSTMSS_BF16)
        return fail(LSTMSS_ERR_UNSUPPORTED, "unknown dtype %d", d->dtype);
    if (d->act < LSTMSS_ACT_NONE || d->act > LSTMSS_ACT_SILU)
        return fail(LSTMSS_ERR_INVALID_ARG, "unknown activation %d", d->act);
    // rows of an operand and offsets within a tile fit 32 bits, the packing
    // grid (a work-group for 64 x 64 elements of each operand) 2^32 threads
    const int64_t J = (int64_t)d->T * d->B, m20 = (int64_t)1 << 20, m32 = (int64_t)1 << 32;
    if (J > m20 || d->K > m20 || d->N > m20 || J * d->K >= m32 || J * d->N >= m32 ||
        (int64_t)d->N * d->K >= m32)
        return fail(LSTMSS_ERR_UNSUPPORTED, "sizes too large");
    return LSTMSS_OK;
}

int32_t check_orth(const lstmss_orth *d) {
    if (!d)
        return fail(LSTMSS_ERR_INVALID_ARG, "sizes are NULL");
    if (d->rows < 1 || d->cols < 1 || d->blocks < 1)
        return fail(LSTMSS_ERR_INVALID_ARG, "sizes must be positive (rows=%d cols=%d blocks=%d)", d->rows,
                    d->cols, d->blocks);
    if (d->dtype != LSTMSS_F32 && d->dtype != LSTMSS_BF16)
        return fail(LSTMSS_ERR_UNSUPPORTED, "unknown dtype %d", d->dtype);
    if (d->rows > 1 << 15 || d->cols > 1 << 15 || d->blocks > 256 ||
        (int64_t)d->blocks * d->rows * d->cols >= (int64_t)1 << 31)
        return fail(LSTMSS_ERR_UNSUPPORTED, "sizes too large");
    if (d->steps < 1 || d->steps > 100)
        return fail(LSTMSS_ERR_INVALID_ARG, "steps=%d must be in [1, 100]", d->steps);
    if (!std::isfinite(d->a) || !std::isfinite(d->b) || !std::isfinite(d->c))
        return fail(LSTMSS_ERR_INVALID_ARG, "coefficients (%g, %g, %g) must be finite", (double)d->a,
                    (double)d->b, (double)d->c);
    return LSTMSS_OK;
}

int32_t muon_call(const char *what, const lstmss_orth *d, MuonArgs &a, void *ws, size_t ws_bytes,
                  void *stream) {
    a.R = d->rows;
    a.C = d->cols;
    a.blocks = d->blocks;
    a.bf16 = d->dtype == LSTMSS_BF16;
    a.steps = d->steps;
    a.a = d->a;
    a.b = d->b;
    a.c = d->c;
    a.eps = 1e-7f;
    const size_t need = muon_ws(a.R, a.C, a.blocks);
    if (int32_t rc = check_ws(ws, ws_bytes, need))
        return rc;
    const int64_t n = (int64_t)a.blocks * a.R * a.C, es = size_of(d->dtype);
    if (a.W ? meets({{a.Wo, n * es}, {a.Mo, n * 4}, {ws, (int64_t)need}},
                    {or_out(a.W, a.Wo, n * es), or_out(a.M, a.Mo, n * 4), {a.dW, n * 4}})
            : meets({{a.Wo, n * es}, {ws, (int64_t)need}}, {or_out(a.dW, a.Wo, n * es)}))
        return fail(LSTMSS_ERR_INVALID_ARG,
                    "an output may be its input (W_out W, M_out M, X_out G), but must overlap nothing else");
    a.ws = ws;
    return enqueue(what, stream, [&] { return launch_muon(a, (hipStream_t)stream); });
}

int32_t check_beams(const lstmss_beams *d) {
    if (!d)
        return fail(LSTMSS_ERR_INVALID_ARG, "sizes are NULL");
    if (d->S < 1 || d->K < 1 || d->V < 1)
        return fail(LSTMSS_ERR_INVALID_ARG, "sizes must be positive (S=%d K=%d V=%d)", d->S, d->K, d->V);
    if (d->dtype != LSTMSS_F32 && d->dtype != LSTMSS_BF16)
        return fail(LSTMSS_ERR_UNSUPPORTED, "unknown dtype %d", d->dtype);
    if (d->K > 32 || d->V > 1 << 26 || (int64_t)d->S * d->K > 1 << 20 ||
        (int64_t)d->K * d->V >= (int64_t)1 << 31)
        return fail(LSTMSS_ERR_UNSUPPORTED, "sizes too large");
    return LSTMSS_OK;
}

// N columns of sequences of K beams.
int32_t check_columns(int64_t N, int32_t K) {
    if (N < 1 || K < 1 || N % K != 0)
        return fail(LSTMSS_ERR_INVALID_ARG, "%lld columns are not sequences of %d beams", (long long)N, K);
    if (N > 1 << 20)
        return fail(LSTMSS_ERR_UNSUPPORTED, "sizes too large");
    return LSTMSS_OK;
}

int32_t check_some_ws(const void *ws, size_t have, size_t need) {
    return need ? check_ws(ws, have, need) : LSTMSS_OK;
}

} // namespace

extern "C" {

int64_t lstmss_linear_workspace_bytes(const lstmss_linear_dims *d) {
    if (int32_t rc = check_linear(d))
        return rc;
    return (int64_t)linear_ws(d->T, d->B, d->K, d->N, d->dtype == LSTMSS_BF16);
}

int32_t lstmss_linear(const lstmss_linear_dims *d, const void *x, const void *W, const float *b,
                      const void *res, void *z, void *y, void *ws, size_t ws_bytes, void *stream) {
    if (int32_t rc = check_linear(d))
        return rc;
    if (!x || !W || !y)
        return fail(LSTMSS_ERR_INVALID_ARG, "a required pointer is NULL");
    LinearArgs a;
    a.T = d->T;
    a.B = d->B;
    a.K = d->K;
    a.N = d->N;
    a.act = d->act;
    a.bf16 = d->dtype == LSTMSS_BF16;
    const size_t need = linear_ws(a.T, a.B, a.K, a.N, a.bf16);
    if (int32_t rc = check_some_ws(ws, ws_bytes, need))
        return rc;
    const int64_t es = size_of(d->dtype), J = (int64_t)a.T * a.B, out = J * a.N * es;
    if (meets({{y, out}, {z, out}, {ws, (int64_t)need}},
              {{x, J * a.K * es}, {W, (int64_t)a.N * a.K * es}, {b, a.N * 4l}, or_out(res, y, out)}))
        return fail(LSTMSS_ERR_INVALID_ARG, "y, z and ws must overlap no input (y may be res) and not each other");
    a.x = x;
    a.W = W;
    a.b = b;
    a.res = res;
    a.z = z;
    a.y = y;
    a.ws = ws;
    return enqueue("linear", stream, [&] { return launch_linear(a, (hipStream_t)stream); });
}

int64_t lstmss_linear_grad_workspace_bytes(const lstmss_linear_dims *d, int32_t dy_dtype) {
    if (int32_t rc = check_linear(d))
        return rc;
    if (dy_dtype != LSTMSS_F32 && dy_dtype != d->dtype)
        return fail(LSTMSS_ERR_UNSUPPORTED, "dY's dtype %d is neither fp32 nor the storage type", dy_dtype);
    return (int64_t)linear_grad_ws(d->T, d->B, d->K, d->N, d->dtype == LSTMSS_BF16, dy_dtype == LSTMSS_BF16,
                                   d->act);
}

int32_t lstmss_linear_grad(const lstmss_linear_dims *d, const void *x, const void *W, const void *z,
                           const void *dY, int32_t dy_dtype, int32_t accumulate, float *dX,
                           float *dW, float *db, void *ws, size_t ws_bytes, void *stream) {
    if (int32_t rc = check_linear(d))
        return rc;
    if (dy_dtype != LSTMSS_F32 && dy_dtype != d->dtype)
        return fail(LSTMSS_ERR_UNSUPPORTED, "dY's dtype %d is neither fp32 nor the storage type", dy_dtype);
    if (!dY || (dW && !x) || (dX && !W) || (!dX && !dW && !db))
        return fail(LSTMSS_ERR_INVALID_ARG, "a required pointer is NULL");
    if ((d->act != LSTMSS_ACT_NONE) != (z != nullptr))
        return fail(LSTMSS_ERR_INVALID_ARG, "z is needed where there is an activation, and only there");
    LinearGradArgs a;
    a.T = d->T;
    a.B = d->B;
    a.K = d->K;
    a.N = d->N;
    a.act = d->act;
    a.bf16 = d->dtype == LSTMSS_BF16;
    a.dy_bf16 = dy_dtype == LSTMSS_BF16;
    const size_t need = linear_grad_ws(a.T, a.B, a.K, a.N, a.bf16, a.dy_bf16, a.act);
    if (int32_t rc = check_some_ws(ws, ws_bytes, need))
        return rc;
    const int64_t es = size_of(d->dtype), J = (int64_t)a.T * a.B, NK = (int64_t)a.N * a.K;
    if (meets({{dX, J * a.K * 4}, {dW, NK * 4}, {db, a.N * 4l}, {ws, (int64_t)need}},
              {{x, J * a.K * es}, {W, NK * es}, {z, J * a.N * es}, {dY, J * a.N * size_of(dy_dtype)}}))
        return fail(LSTMSS_ERR_INVALID_ARG, "gradients and ws must overlap no input and not each other");
    a.x = x;
    a.W = W;
    a.z = z;
    a.dY = dY;
    a.accumulate = accumulate != 0;
    a.dX = dX;
    a.dW = dW;
    a.db = db;
    a.ws = ws;
    return enqueue("linear_grad", stream, [&] { return launch_linear_grad(a, (hipStream_t)stream); });
}

int64_t lstmss_muon_workspace_bytes(const lstmss_orth *d) {
    if (int32_t rc = check_orth(d))
        return rc;
    return (int64_t)muon_ws(d->rows, d->cols, d->blocks);
}

int32_t lstmss_orthogonalize(const lstmss_orth *d, const float *G, float *X_out, void *ws,
                             size_t ws_bytes, void *stream) {
    if (int32_t rc = check_orth(d))
        return rc;
    if (d->dtype != LSTMSS_F32)
        return fail(LSTMSS_ERR_UNSUPPORTED, "dtype %d is not fp32", d->dtype);
    if (!G || !X_out)
        return fail(LSTMSS_ERR_INVALID_ARG, "a required pointer is NULL");
    MuonArgs a = {};
    a.dW = G;
    a.Wo = X_out;
    return muon_call("orthogonalize", d, a, ws, ws_bytes, stream);
}

int32_t lstmss_muon_update(const lstmss_orth *d, const lstmss_muon *p, const void *W, const float *M,
                           const float *dW, void *W_out, float *M_out, void *ws, size_t ws_bytes,
                           void *stream) {
    if (int32_t rc = check_orth(d))
        return rc;
    if (!p || !W || !M || !dW || !W_out || !M_out)
        return fail(LSTMSS_ERR_INVALID_ARG, "a required pointer is NULL");
    if (!std::isfinite(p->lr) || !std::isfinite(p->decay) || !std::isfinite(p->scale))
        return fail(LSTMSS_ERR_INVALID_ARG, "lr=%g, decay=%g and scale=%g must be finite", (double)p->lr,
                    (double)p->decay, (double)p->scale);
    if (!(p->momentum >= 0.f) || !(p->momentum < 1.f))
        return fail(LSTMSS_ERR_INVALID_ARG, "momentum=%g must be in [0, 1)", (double)p->momentum);
    MuonArgs a = {};
    a.lr = p->lr;
    a.mu = p->momentum;
    a.decay = p->decay;
    a.scale = p->scale;
    a.nesterov = p->nesterov != 0;
    a.W = W;
    a.M = M;
    a.dW = dW;
    a.Wo = W_out;
    a.Mo = M_out;
    return muon_call("muon_update", d, a, ws, ws_bytes, stream);
}

int64_t lstmss_beam_workspace_bytes(const lstmss_beams *d) {
    if (int32_t rc = check_beams(d))
        return rc;
    return (int64_t)beam_ws(d->S, d->K, d->V);
}

int32_t lstmss_beam_step(const lstmss_beams *d, const void *logits, const float *scores, int32_t eos,
                         const int32_t *done, float *scores_out, int32_t *tokens, int32_t *parents,
                         int32_t *done_out, void *ws, size_t ws_bytes, void *stream) {
    if (int32_t rc = check_beams(d))
        return rc;
    if (!logits || !scores || !scores_out || !tokens || !parents)
        return fail(LSTMSS_ERR_INVALID_ARG, "a required pointer is NULL");
    if (eos < -1 || eos >= d->V)
        return fail(LSTMSS_ERR_INVALID_ARG, "eos=%d must be -1 or in [0, %d)", eos, d->V);
    if (eos < 0 && (done || done_out))
        return fail(LSTMSS_ERR_INVALID_ARG, "no beam is finished without an eos");
    const size_t need = beam_ws(d->S, d->K, d->V);
    if (int32_t rc = check_ws(ws, ws_bytes, need))
        return rc;
    const int64_t N = (int64_t)d->S * d->K, n = N * 4;
    if (meets({{scores_out, n}, {tokens, n}, {parents, n}, {done_out, n}, {ws, (int64_t)need}},
              {{logits, d->V * N * size_of(d->dtype)}, or_out(scores, scores_out, n), or_out(done, done_out, n)}))
        return fail(LSTMSS_ERR_INVALID_ARG,
                    "scores_out may be scores and done_out done, but outputs must overlap nothing else");
    BeamArgs a;
    a.S = d->S;
    a.K = d->K;
    a.V = d->V;
    a.bf16 = d->dtype == LSTMSS_BF16;
    a.eos = eos;
    a.logits = logits;
    a.scores = scores;
    a.done = done;
    a.scores_out = scores_out;
    a.tokens = tokens;
    a.parents = parents;
    a.done_out = done_out;
    a.ws = ws;
    return enqueue("beam_step", stream, [&] { return launch_beam(a, (hipStream_t)stream); });
}

int32_t lstmss_beam_reorder(int64_t rows, int32_t N, int32_t K, int32_t dtype, const int32_t *parents,
                            const void *x, void *out, void *stream) {
    if (int32_t rc = check_columns(N, K))
        return rc;
    if (rows < 1)
        return fail(LSTMSS_ERR_INVALID_ARG, "rows=%lld must be positive", (long long)rows);
    if (rows >= (int64_t)1 << 40)
        return fail(LSTMSS_ERR_UNSUPPORTED, "sizes too large");
    if (dtype != LSTMSS_F32 && dtype != LSTMSS_BF16)
        return fail(LSTMSS_ERR_UNSUPPORTED, "unknown dtype %d", dtype);
    if (!parents || !x || !out)
        return fail(LSTMSS_ERR_INVALID_ARG, "a required pointer is NULL");
    const int64_t bytes = rows * N * size_of(dtype);
    if (meets({{out, bytes}}, {{x, bytes}, {parents, N * 4l}}))
        return fail(LSTMSS_ERR_INVALID_ARG, "out must overlap neither x nor parents");
    return enqueue("beam_reorder", stream, [&] {
        return launch_beam_reorder((long)rows, N, K, dtype == LSTMSS_BF16, parents, x, out, (hipStream_t)stream);
    });
}

int32_t lstmss_beam_trace(int32_t T, int32_t N, int32_t K, const int32_t *tokens,
                          const int32_t *parents, int32_t *out, void *stream) {
    if (int32_t rc = check_columns(N, K))
        return rc;
    if (T < 1)
        return fail(LSTMSS_ERR_INVALID_ARG, "T=%d must be positive", T);
    if (!tokens || !parents || !out)
        return fail(LSTMSS_ERR_INVALID_ARG, "a required pointer is NULL");
    const int64_t bytes = (int64_t)T * N * 4;
    if (meets({{out, bytes}}, {{tokens, bytes}, {parents, bytes}}))
        return fail(LSTMSS_ERR_INVALID_ARG, "out must overlap neither tokens nor parents");
    return enqueue("beam_trace", stream,
                   [&] { return launch_beam_trace(T, N, K, tokens, parents, out, (hipStream_t)stream); });
}

} // extern "C"
