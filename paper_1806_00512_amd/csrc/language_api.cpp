// Host side of the language-model operators: argument checks and launches.
//
// One translation unit with the layers' entry points: the calling thread's
// error message and the timing records are theirs, and these calls set them too.
#include "lstmss_api.cpp"

#include "language.h"

namespace {

// Runs f(), which enqueues a call's kernels, under the timing hooks.
template <class F>
int32_t enqueue(const char *what, void *stream, F &&f) {
    const hipError_t e = timed(LSTMSS_KERNEL_AUX, (hipStream_t)stream, f);
    if (e != hipSuccess)
        return fail(LSTMSS_ERR_HIP, "%s failed: %s", what, hipGetErrorString(e));
    return LSTMSS_OK;
}

int32_t check_tokens(const lstmss_tokens *d, bool dtype) {
    if (!d)
        return fail(LSTMSS_ERR_INVALID_ARG, "sizes are NULL");
    if (d->T < 1 || d->B < 1 || d->I < 1 || d->V < 1)
        return fail(LSTMSS_ERR_INVALID_ARG, "sizes must be positive (T=%d B=%d I=%d V=%d)", d->T,
                    d->B, d->I, d->V);
    if (dtype && d->dtype != LSTMSS_F32 && d->dtype != LSTMSS_BF16)
        return fail(LSTMSS_ERR_UNSUPPORTED, "unknown dtype %d", d->dtype);
    // indices within a step and row numbers fit 32 bits; grids (a work-group for
    // each step and 40 or more of its columns, and for 64 features of these, or
    // for 16 rows of the table; 256 threads for 16 tokens) stay below 2^32 threads
    const int64_t N = (int64_t)d->T * d->B, m31 = (int64_t)1 << 31;
    const int64_t steps = (int64_t)d->T * (d->B / 33 + 1), tiles = steps * (d->I / 64 + 1);
    if (N > ((int64_t)1 << 28) - 16 || d->V > 1 << 26 || (int64_t)d->V * d->B >= m31 || (int64_t)d->V * d->I >= m31 ||
        (int64_t)d->I * d->B >= m31 || tiles >= (int64_t)1 << 23)
        return fail(LSTMSS_ERR_UNSUPPORTED, "sizes too large");
    return LSTMSS_OK;
}

int32_t check_drop(const lstmss_drop *d, DropArgs *a) {
    *a = DropArgs{0, 1.f, 0, 0, 0, 0};
    if (!d)
        return LSTMSS_OK;
    if (!(d->p >= 0.f) || !(d->p < 1.f))
        return fail(LSTMSS_ERR_INVALID_ARG, "dropout p=%g must be in [0, 1)", (double)d->p);
    if (d->offset % 8 != 0)
        return fail(LSTMSS_ERR_INVALID_ARG, "dropout offset %llu is not a multiple of 8",
                    (unsigned long long)d->offset);
    if (d->period < 0)
        return fail(LSTMSS_ERR_INVALID_ARG, "dropout period %lld is negative", (long long)d->period);
    const double thr = std::fmin(std::nearbyint((double)d->p * 65536.0), 65535.0);
    a->thr = (uint32_t)thr;
    a->scale = (float)(65536.0 / (65536.0 - thr));
    a->key0 = (uint32_t)d->seed;
    a->key1 = (uint32_t)(d->seed >> 32);
    a->counter = d->offset / 8;
    a->period = (long)d->period;
    return LSTMSS_OK;
}

int32_t check_ws(const void *ws, size_t have, size_t need) {
    if (!ws || have < need)
        return fail(LSTMSS_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws ? have : (size_t)0, need);
    if ((uintptr_t)ws % 16 != 0)
        return fail(LSTMSS_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
    return LSTMSS_OK;
}

int32_t loss_call(const char *what, const lstmss_tokens *d, LossArgs &a, void *ws, size_t ws_bytes,
                  void *stream) {
    if (!a.logits || !a.targets)
        return fail(LSTMSS_ERR_INVALID_ARG, "a required pointer is NULL");
    if (!std::isfinite(a.scale))
        return fail(LSTMSS_ERR_INVALID_ARG, "scale %g is not finite", (double)a.scale);
    a.T = d->T;
    a.B = d->B;
    a.V = d->V;
    a.bf16 = d->dtype == LSTMSS_BF16;
    if (int32_t rc = check_ws(ws, ws_bytes, loss_ws(a.T, a.B, a.V, a.bf16)))
        return rc;
    a.ws = ws;
    return enqueue(what, stream, [&] { return launch_loss(a, (hipStream_t)stream); });
}

} // namespace

extern "C" {

int32_t lstmss_dropout(int64_t n, int32_t dtype, const lstmss_drop *drop, const void *x, void *y,
                       void *stream) {
    if (n < 1)
        return fail(LSTMSS_ERR_INVALID_ARG, "n=%lld must be positive", (long long)n);
    if (n >= (int64_t)1 << 40)
        return fail(LSTMSS_ERR_UNSUPPORTED, "sizes too large");
    if (dtype != LSTMSS_F32 && dtype != LSTMSS_BF16)
        return fail(LSTMSS_ERR_UNSUPPORTED, "unknown dtype %d", dtype);
    if (!drop || !x || !y)
        return fail(LSTMSS_ERR_INVALID_ARG, "a required pointer is NULL");
    DropArgs a;
    if (int32_t rc = check_drop(drop, &a))
        return rc;
    return enqueue("dropout", stream, [&] {
        return launch_dropout(a, (long)n, x, y, dtype == LSTMSS_BF16, (hipStream_t)stream);
    });
}

int32_t lstmss_embed(const lstmss_tokens *d, const void *E, const int32_t *tokens, float scale,
                     const lstmss_drop *drop, void *x, void *stream) {
    if (int32_t rc = check_tokens(d, true))
        return rc;
    if (!E || !tokens || !x)
        return fail(LSTMSS_ERR_INVALID_ARG, "a required pointer is NULL");
    // (the zeros of padding are scaled too)
    if (!std::isfinite(scale))
        return fail(LSTMSS_ERR_INVALID_ARG, "scale %g is not finite", (double)scale);
    EmbedArgs a;
    if (int32_t rc = check_drop(drop, &a.drop))
        return rc;
    a.T = d->T;
    a.B = d->B;
    a.I = d->I;
    a.V = d->V;
    a.tokens = tokens;
    a.scale = scale;
    a.E = E;
    a.x = x;
    return enqueue("embed", stream,
                   [&] { return launch_embed(a, d->dtype == LSTMSS_BF16, (hipStream_t)stream); });
}

int64_t lstmss_embed_grad_workspace_bytes(const lstmss_tokens *d) {
    if (int32_t rc = check_tokens(d, false))
        return rc;
    return (int64_t)embed_grad_ws(d->T, d->B, d->I, d->V);
}

int32_t lstmss_embed_grad(const lstmss_tokens *d, const int32_t *tokens, const float *dX,
                          float scale, const lstmss_drop *drop, int32_t accumulate, float *dE,
                          void *ws, size_t ws_bytes, void *stream) {
    if (int32_t rc = check_tokens(d, false))
        return rc;
    if (!tokens || !dX || !dE)
        return fail(LSTMSS_ERR_INVALID_ARG, "a required pointer is NULL");
    EmbedGradArgs a;
    if (int32_t rc = check_drop(drop, &a.drop))
        return rc;
    if (int32_t rc = check_ws(ws, ws_bytes, embed_grad_ws(d->T, d->B, d->I, d->V)))
        return rc;
    a.T = d->T;
    a.B = d->B;
    a.I = d->I;
    a.V = d->V;
    a.tokens = tokens;
    a.scale = scale;
    a.dX = dX;
    a.accumulate = accumulate != 0;
    a.dE = dE;
    a.ws = ws;
    return enqueue("embed_grad", stream, [&] { return launch_embed_grad(a, (hipStream_t)stream); });
}

int64_t lstmss_loss_workspace_bytes(const lstmss_tokens *d) {
    if (int32_t rc = check_tokens(d, true))
        return rc;
    return (int64_t)loss_ws(d->T, d->B, d->V, d->dtype == LSTMSS_BF16);
}

int32_t lstmss_token_logp(const lstmss_tokens *d, const void *logits, const int32_t *targets,
                          float *logp, void *ws, size_t ws_bytes, void *stream) {
    if (int32_t rc = check_tokens(d, true))
        return rc;
    if (!logp)
        return fail(LSTMSS_ERR_INVALID_ARG, "a required pointer is NULL");
    LossArgs a = {};
    a.mode = LOSS_LOGP;
    a.logits = logits;
    a.targets = targets;
    a.logp = logp;
    return loss_call("token_logp", d, a, ws, ws_bytes, stream);
}

int32_t lstmss_xent(const lstmss_tokens *d, const void *logits, const int32_t *targets,
                    const float *weights, float scale, float *loss, float *logp, void *dlogits,
                    void *ws, size_t ws_bytes, void *stream) {
    if (int32_t rc = check_tokens(d, true))
        return rc;
    LossArgs a = {};
    a.mode = LOSS_XENT;
    a.logits = logits;
    a.targets = targets;
    a.weights = weights;
    a.scale = scale;
    a.loss = loss;
    a.logp = logp;
    a.dlogits = dlogits;
    return loss_call("xent", d, a, ws, ws_bytes, stream);
}

int32_t lstmss_policy_loss(const lstmss_tokens *d, const lstmss_policy *p, const void *logits,
                           const int32_t *targets, const float *logp_old, const float *logp_ref,
                           const float *adv, const float *weights, float *loss, float *logp,
                           void *dlogits, void *ws, size_t ws_bytes, void *stream) {
    if (int32_t rc = check_tokens(d, true))
        return rc;
    if (!p || !adv)
        return fail(LSTMSS_ERR_INVALID_ARG, "a required pointer is NULL");
    if (!(p->clip_low >= 0.f) || !(p->clip_low <= 1.f) || !(p->clip_high >= 0.f) ||
        !std::isfinite(p->clip_high))
        return fail(LSTMSS_ERR_INVALID_ARG, "clip range (%g, %g): low in [0, 1], high >= 0",
                    (double)p->clip_low, (double)p->clip_high);
    if (!(p->kl >= 0.f) || !std::isfinite(p->kl) || (p->kl > 0.f && !logp_ref))
        return fail(LSTMSS_ERR_INVALID_ARG, "kl=%g must be >= 0, and 0 without logp_ref",
                    (double)p->kl);
    LossArgs a = {};
    a.mode = LOSS_POLICY;
    a.logits = logits;
    a.targets = targets;
    a.weights = weights;
    a.old_logp = logp_old;
    a.ref_logp = p->kl > 0.f ? logp_ref : nullptr;
    a.adv = adv;
    a.clip_low = p->clip_low;
    a.clip_high = p->clip_high;
    a.kl = p->kl;
    a.scale = p->scale;
    a.loss = loss;
    a.logp = logp;
    a.dlogits = dlogits;
    return loss_call("policy_loss", d, a, ws, ws_bytes, stream);
}

} // extern "C"
