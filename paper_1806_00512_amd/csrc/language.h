// Launchers of the language-model operators (embedding, dropout, vocabulary
// losses), called by language_api.cpp.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lstmss {

// Dropout as the kernels take it: threshold of the 16 bits (0 = keep all),
// scale of what is kept, key, first counter, period (0 = none).
struct DropArgs {
    uint32_t thr;
    float scale;
    uint32_t key0, key1;
    uint64_t counter;
    long period;
};

struct EmbedArgs {
    int T, B, I, V;
    const int32_t *tokens; // [T][B]
    float scale;
    DropArgs drop;
    const void *E; // [V][I]
    void *x;       // [T][I][B]
};

struct EmbedGradArgs {
    int T, B, I, V;
    const int32_t *tokens; // [T][B]
    float scale;
    DropArgs drop;
    const float *dX; // [T][I][B]
    bool accumulate;
    float *dE; // [V][I]
    void *ws;
};

// per-token terms of a loss
enum { LOSS_LOGP = 0, LOSS_XENT = 1, LOSS_POLICY = 2 };

struct LossArgs {
    int T, B, V;
    int mode;
    bool bf16;
    const void *logits; // [T][V][B]
    const int32_t *targets;
    const float *weights, *old_logp, *ref_logp, *adv; // [T][B] or NULL
    float clip_low, clip_high, kl, scale;
    float *loss, *logp; // [1], [T][B], or NULL
    void *dlogits;      // [T][V][B] or NULL
    void *ws;
};

hipError_t launch_dropout(const DropArgs &d, long n, const void *x, void *y, bool bf16,
                          hipStream_t s);
hipError_t launch_embed(const EmbedArgs &a, bool bf16, hipStream_t s);
size_t embed_grad_ws(int T, int B, int I, int V);
hipError_t launch_embed_grad(const EmbedGradArgs &a, hipStream_t s);
size_t loss_ws(int T, int B, int V, bool bf16);
hipError_t launch_loss(const LossArgs &a, hipStream_t s);

} // namespace lstmss
