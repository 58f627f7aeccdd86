"""Performance cases of the language-model operators around the LSTM layers.

What stands below the first layer and above the last one when the layers train
a language model, in the package's batch-last layouts:

  embed        x[t][i][b] = scale * E[tokens[t][b]][i], with dropout on the way
  embed_grad   dE[v][i] = scale * the sum of dX[t][i][b] over the (t, b) with token v
  dropout      elements kept or dropped by a counter-based generator; no stored mask
  token_logp   log softmax over the vocabulary of logits [T][V][B], at the target
  xent         -scale * sum of w * logp, and its gradient in the logits
  policy_loss  clipped policy loss with a KL term, and its gradient in the logits

Every case is one pass through one of them.  Sizes are those of the package's
workloads (paper_1806_00512_amd/inputs.py), with a vocabulary beside them.

Tokens follow a Zipf law (token v with weight 1 / (v + 1)), and the sequences
of a batch have different lengths: what lies past a sequence's end has token or
target -1 and takes no part.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one token of one sequence, as a server feeds it: latency alone
        {"name": "embed_one", "op": "embed", "dtype": "f32", "T": 1, "B": 1, "I": 650, "V": 10000,
         "p": 0.0},
        # the largest layer's input, bf16, with dropout on the embedding
        {"name": "embed_big", "op": "embed", "dtype": "bf16", "T": 100, "B": 256, "I": 4096,
         "V": 32000, "p": 0.1},
        # word language model (650 features, batch 20): launches and the sort count
        {"name": "embed_grad_lm", "op": "embed_grad", "dtype": "f32", "T": 35, "B": 20, "I": 650,
         "V": 10000, "p": 0.5},
        # sequence-to-sequence encoder: long runs of the frequent tokens
        {"name": "embed_grad_enc", "op": "embed_grad", "dtype": "f32", "T": 50, "B": 128, "I": 2048,
         "V": 32000, "p": 0.0},
        # nothing is a multiple of anything
        {"name": "embed_grad_odd", "op": "embed_grad", "dtype": "f32", "T": 37, "B": 33, "I": 1023,
         "V": 5003, "p": 0.25},
        # between the two layers of the word language model
        {"name": "dropout_lm", "op": "dropout", "dtype": "f32", "T": 35, "B": 20, "I": 650,
         "p": 0.5, "shared": False},
        # on the largest layer's output, one mask for all steps
        {"name": "dropout_big", "op": "dropout", "dtype": "bf16", "T": 100, "B": 256, "I": 4096,
         "p": 0.1, "shared": True},
        # scores of one step's tokens, as a server asks for them
        {"name": "logp_one", "op": "token_logp", "dtype": "f32", "T": 1, "B": 16, "V": 10000},
        # word language model: loss and gradient of a training step
        {"name": "xent_lm", "op": "xent", "dtype": "f32", "T": 35, "B": 20, "V": 10000},
        # encoder-sized batch over a large vocabulary, bf16 logits
        {"name": "xent_big", "op": "xent", "dtype": "bf16", "T": 50, "B": 128, "V": 32000},
        # policy update of an odd-sized batch
        {"name": "policy_odd", "op": "policy_loss", "dtype": "f32", "T": 37, "B": 33, "V": 5003},
        # policy update of the two-layer model's batch
        {"name": "policy_mid", "op": "policy_loss", "dtype": "bf16", "T": 35, "B": 64, "V": 10000},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: every operator, both types, 1 to 100 steps, batches of 1
    to 256, 64 to 4096 features, vocabularies of 1000 to 32000."""
    while True:
        c = {"op": rng.choice(["embed", "embed_grad", "dropout", "token_logp", "xent",
                               "policy_loss"]),
             "dtype": rng.choice(["f32", "bf16"])}
        c["T"], c["B"] = _log_int(rng, 1, 100), _log_int(rng, 1, 256)
        I, V = _log_int(rng, 64, 4096), _log_int(rng, 1000, 32000)
        if rng.random() < 0.4:  # whole tiles
            c["B"], I = max(8, c["B"] // 8 * 8), max(64, I // 64 * 64)
        if c["op"] in ("embed", "embed_grad", "dropout"):
            c["I"] = I
            c["p"] = rng.choice([0.0, 0.1, 0.25, 0.5]) if c["op"] != "dropout" else \
                rng.choice([0.1, 0.3, 0.5, 0.65])
        if c["op"] == "embed_grad":
            c["dtype"] = "f32"  # gradients are fp32 whatever the embedding's type
        if c["op"] == "dropout":
            c["shared"] = rng.random() < 0.5
        else:
            c["V"] = V
        if work(c)["bytes"] <= work(listed()[9])["bytes"]:
            return c


# ---------------------------------------------------------------- inputs

def _lengths(T, B, g):
    """Lengths of the batch's sequences: half of them whole, the others shorter."""
    part = torch.rand(B, generator=g, device=DEV)
    n = torch.where(part < 0.5, torch.ones_like(part), part) * T
    return n.ceil().to(torch.int64).clamp(1, T)


def _tokens(T, B, V, g):
    """[T][B] int32 by a Zipf law, -1 past a sequence's end."""
    u = torch.rand((T, B), generator=g, device=DEV, dtype=torch.float64)
    tok = (float(V) ** u - 1.0).to(torch.int32).clamp(0, V - 1)
    past = torch.arange(T, device=DEV)[:, None] >= _lengths(T, B, g)[None, :]
    return tok.masked_fill_(past, -1).contiguous()


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt, T, B = DTYPES[case["dtype"]], case["T"], case["B"]
    s = {"case": case}

    def normal(shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, device=DEV).normal_(0.0, std, generator=g).to(dtype)

    if "p" in case:
        # a training program numbers its draws: `offset` is what earlier calls took
        s["p"], s["seed"], s["offset"] = case["p"], 0x9E3779B97F4A7C15 ^ (seed * 65537), 8 * seed
        s["period"] = 0
    op = case["op"]
    if op == "embed":
        I, V = case["I"], case["V"]
        s["scale"] = math.sqrt(I)
        s["E"] = normal((V, I), 1.0 / math.sqrt(I), dt)
        s["tokens"] = _tokens(T, B, V, g)
        s["x"] = torch.empty((T, I, B), dtype=dt, device=DEV)
    elif op == "embed_grad":
        I, V = case["I"], case["V"]
        s["scale"] = math.sqrt(I)
        s["dX"] = normal((T, I, B), 0.01)
        s["tokens"] = _tokens(T, B, V, g)
        s["dE"] = torch.empty((V, I), device=DEV)
    elif op == "dropout":
        s["x"] = torch.tanh(normal((T, case["I"], B))).to(dt)
        s["y"] = torch.empty_like(s["x"])
        s["period"] = case["I"] * B if case["shared"] else 0
    else:
        V = case["V"]
        # logits of a trained model: frequent tokens stand higher
        x = normal((T, V, B), 2.0)
        x -= 0.5 * torch.log(torch.arange(1, V + 1, device=DEV).float())[None, :, None]
        s["logits"] = x.to(dt)
        del x
        s["targets"] = _tokens(T, B, V, g)
        s["logp"] = torch.empty((T, B), device=DEV)
        s["scale"] = 1.0 / B
        if op != "token_logp":
            s["loss"] = torch.empty(1, device=DEV)
            s["dlogits"] = torch.empty_like(s["logits"])
        if op == "xent":
            # weights of the sequences, as for samples of several sources
            s["weights"] = (0.5 + torch.rand((1, B), generator=g, device=DEV)).repeat(T, 1)
        if op == "policy_loss":
            s["clip_low"], s["clip_high"], s["kl"] = 0.2, 0.25, 0.05
            now = torch.stack([z.float().logsumexp(0) for z in s["logits"]])
            at = s["targets"].clamp(min=0).long()
            now = s["logits"].gather(1, at[:, None]).float()[:, 0] - now
            # log ratios, none so near the clip's two corners that a rounding
            # decides on which side it is
            r = normal((T, B), 0.2)
            for corner in (math.log(1.0 - s["clip_low"]), math.log(1.0 + s["clip_high"])):
                r += torch.where((r - corner).abs() < 1e-3, 2e-3, 0.0)
            s["old"] = now - r
            s["ref"] = now + normal((T, B), 0.3)
            # one advantage for each sequence, a little above zero on average
            s["adv"] = (normal((1, B)) + 0.3).repeat(T, 1)
    return s


# ---------------------------------------------------------------- plain forms

def _philox(counter, seed):
    """Philox4x32-10 (Salmon et al., 2011): four 32-bit words for each counter."""
    low = 0xFFFFFFFF
    c = [counter & low, counter >> 32, torch.zeros_like(counter), torch.zeros_like(counter)]
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57  # wraps: the low 64 bits are what counts
        c = [((b >> 32) & low) ^ c[1] ^ k0, b & low, ((a >> 32) & low) ^ c[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c


def _drop(x, s):
    """x with dropout, in fp32: element e takes 16 of the 128 bits of counter (offset + e) / 8,
    e modulo the period where there is one, and is kept where they are p * 65536 or more."""
    thr = int(round(s["p"] * 65536.0))
    if thr == 0:
        return x
    n = s["period"] or x.numel()
    at = torch.arange(-(-n // 8), device=x.device) + s["offset"] // 8
    words = _philox(at, s["seed"])
    bits = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], 1).reshape(-1)[:n]
    keep = (bits >= thr).expand(x.numel() // n, n).reshape(x.shape)
    return torch.where(keep, x * (65536.0 / (65536.0 - thr)), 0.0)


def _plain_embed(s):
    tok = s["tokens"]
    x = s["E"][tok.clamp(min=0).long()].float() * s["scale"]
    x = torch.where((tok >= 0)[..., None], x, 0.0).permute(0, 2, 1).contiguous()
    return _drop(x, s).to(s["E"].dtype)


def _plain_embed_grad(s):
    tok = s["tokens"].reshape(-1)
    g = _drop(s["dX"], s).permute(0, 2, 1).reshape(tok.numel(), -1)
    dE = torch.zeros_like(s["dE"])
    return dE.index_add_(0, tok[tok >= 0].long(), g[tok >= 0] * s["scale"])


def _plain_logp(s):
    """(log probabilities of the targets, 0 where there is none; softmax; targets; mask)."""
    x = s["logits"].float()
    e = torch.exp(x - x.amax(1, keepdim=True))
    total = e.sum(1, keepdim=True)
    there = s["targets"] >= 0
    at = s["targets"].clamp(min=0).long()[:, None]
    logp = x.gather(1, at) - x.amax(1, keepdim=True) - torch.log(total)
    return torch.where(there, logp[:, 0], 0.0), e.div_(total), at, there


def _plain_dlogits(s, dlogp, soft, at):
    g = soft.mul_(-dlogp[:, None])
    g.scatter_add_(1, at, dlogp[:, None])
    return g.to(s["logits"].dtype)


def _plain_xent(s):
    logp, soft, at, there = _plain_logp(s)
    w = torch.where(there, s["weights"], 0.0) * s["scale"]
    return {"loss": -(w * logp).sum().reshape(1), "logp": logp,
            "dlogits": _plain_dlogits(s, -w, soft, at)}


def _plain_policy(s):
    logp, soft, at, there = _plain_logp(s)
    ratio = torch.exp(logp - s["old"])
    clipped = ratio.clamp(1.0 - s["clip_low"], 1.0 + s["clip_high"])
    gain, held = ratio * s["adv"], clipped * s["adv"]
    d = s["ref"] - logp
    each = -torch.minimum(gain, held) + s["kl"] * (torch.exp(d) - d - 1.0)
    dlogp = -torch.where(gain <= held, gain, 0.0) + s["kl"] * (1.0 - torch.exp(d))
    w = there.float() * s["scale"]
    return {"loss": (w * each).sum().reshape(1), "logp": logp,
            "dlogits": _plain_dlogits(s, w * dlogp, soft, at)}


# ---------------------------------------------------------------- a pass

def _kept(s, size):
    """The workspace that a program keeps beside its buffers."""
    if "ws" not in s:
        s["ws"] = torch.empty(size(), dtype=torch.uint8, device=DEV)
    return s["ws"]


def _own(s):
    import paper_1806_00512_amd.lstmss as L
    op, c = s["case"]["op"], s["case"]
    drop = L.drop(s["p"], s["seed"], s["offset"], s["period"]) if s.get("p") else None
    if op == "embed":
        return L.embed(s["tokens"], s["E"], scale=s["scale"], drop=drop, out=s["x"])
    if op == "embed_grad":
        ws = _kept(s, lambda: L.embed_grad_workspace_bytes(c["T"], c["B"], c["I"], c["V"]))
        return L.embed_grad(s["tokens"], s["dX"], c["V"], scale=s["scale"], drop=drop, dE=s["dE"],
                            ws=ws)
    if op == "dropout":
        return L.dropout(s["x"], drop, out=s["y"])
    ws = _kept(s, lambda: L.loss_workspace_bytes(c["T"], c["B"], c["V"], s["logits"].dtype))
    if op == "token_logp":
        return L.token_logp(s["logits"], s["targets"], logp=s["logp"], ws=ws)
    out = {"loss": s["loss"], "logp": s["logp"], "dlogits": s["dlogits"]}
    if op == "xent":
        return L.xent(s["logits"], s["targets"], weights=s["weights"], scale=s["scale"], out=out,
                      ws=ws)
    return L.policy_loss(s["logits"], s["targets"], s["old"], s["ref"], s["adv"],
                         clip_low=s["clip_low"], clip_high=s["clip_high"], kl=s["kl"],
                         scale=s["scale"], out=out, ws=ws)


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "embed":
        return _plain_embed(state)
    if op == "embed_grad":
        return _plain_embed_grad(state)
    if op == "dropout":
        return _drop(state["x"].float(), state).to(state["x"].dtype)
    if op == "token_logp":
        return _plain_logp(state)[0]
    return _plain_xent(state) if op == "xent" else _plain_policy(state)


def _rows(N, V):
    """Distinct tokens expected among N tokens of the law above, 7 in 8 of which are no padding."""
    v = np.arange(1, V + 1)
    each = np.log1p(1.0 / v) / math.log(V + 1)
    return float((1.0 - (1.0 - each) ** (0.875 * N)).sum())


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    N = case["T"] * case["B"]
    op = case["op"]
    if op == "embed":  # the rows in use, the tokens, x
        return {"bytes": (_rows(N, case["V"]) + N) * case["I"] * es + 4 * N, "flops": N * case["I"]}
    if op == "embed_grad":  # dX, the tokens, all of dE
        return {"bytes": 4 * (N + case["V"]) * case["I"] + 4 * N, "flops": 2 * N * case["I"]}
    if op == "dropout":
        return {"bytes": 2 * es * N * case["I"], "flops": N * case["I"]}
    each = {"token_logp": 2, "xent": 3, "policy_loss": 5}[op]  # fp32 values of a token
    n = N * case["V"]
    if op == "token_logp":
        return {"bytes": es * n + 4 * each * N, "flops": 3 * n}
    return {"bytes": 2 * es * n + 4 * each * N, "flops": 6 * n}


# ---------------------------------------------------------------- 64 bits

def _keep64(s, n):
    """Which of the n mask elements are kept, from the generator's definition on 64-bit words."""
    u = np.uint64
    low, half = u(0xFFFFFFFF), u(32)
    at = np.arange(s["offset"] // 8, s["offset"] // 8 + (n + 7) // 8, dtype=np.uint64)
    x0, x1, x2, x3 = at & low, at >> half, np.zeros_like(at), np.zeros_like(at)
    keys = [s["seed"] % 2**32, s["seed"] // 2**32 % 2**32]
    for r in range(10):
        k0, k1 = (u((k + r * w) % 2**32) for k, w in zip(keys, (0x9E3779B9, 0xBB67AE85)))
        p, q = x0 * u(0xD2511F53), x2 * u(0xCD9E8D57)
        x0, x1, x2, x3 = (q >> half) ^ x1 ^ k0, q & low, (p >> half) ^ x3 ^ k1, p & low
    bits = np.stack([x0, x1, x2, x3], 1).astype("<u4").view("<u2").reshape(-1)[:n]
    return bits >= int(round(s["p"] * 65536.0))


def _drop64(x, s):
    if not s["p"]:
        return x
    n = s["period"] or x.numel()
    keep = torch.from_numpy(_keep64(s, n)).to(x.device)
    x = x.reshape(-1, n) / (1.0 - round(s["p"] * 65536.0) / 65536.0)
    return torch.where(keep[None], x, torch.zeros_like(x))


def exact(case, seed):
    s = prepare(case, seed)
    op, T, B = case["op"], case["T"], case["B"]
    f64 = torch.float64
    if op == "dropout":
        return _drop64(s["x"].to(f64), s).reshape(s["x"].shape)
    if op == "embed":
        x = torch.zeros(s["x"].shape, dtype=f64, device=DEV)
        for t in range(T):
            b = torch.nonzero(s["tokens"][t] >= 0)[:, 0]
            x[t][:, b] = s["E"][s["tokens"][t, b].long()].to(f64).t() * s["scale"]
        return _drop64(x, s).reshape(x.shape)
    if op == "embed_grad":
        g = _drop64(s["dX"].to(f64), s).reshape(s["dX"].shape)
        dE = torch.zeros(s["dE"].shape, dtype=f64, device=DEV)
        for t in range(T):
            b = torch.nonzero(s["tokens"][t] >= 0)[:, 0]
            dE.index_put_((s["tokens"][t, b].long(),), g[t][:, b].t() * s["scale"],
                          accumulate=True)
        return dE
    logp = torch.zeros((T, B), dtype=f64, device=DEV)
    grad = torch.empty(s["logits"].shape, dtype=f64, device=DEV) if op != "token_logp" else None
    loss = torch.zeros((), dtype=f64, device=DEV)
    cols = torch.arange(B, device=DEV)
    for t in range(T):
        lp = torch.log_softmax(s["logits"][t].to(f64), 0)
        tgt = s["targets"][t].long()
        on = tgt >= 0
        row = tgt * on
        logp[t] = lp[row, cols] * on
        if op == "token_logp":
            continue
        if op == "xent":
            d = -s["weights"][t].to(f64)
            loss += (d * logp[t] * on).sum() * s["scale"]
        else:
            r = torch.exp(lp[row, cols] - s["old"][t].to(f64))
            a = s["adv"][t].to(f64)
            top, bottom = 1.0 + s["clip_high"], 1.0 - s["clip_low"]
            shut = ((a > 0) & (r > top)) | ((a < 0) & (r < bottom))
            q = s["ref"][t].to(f64) - lp[row, cols]
            each = -a * torch.where(shut, torch.where(a > 0, top, bottom), r)
            loss += ((each + s["kl"] * (torch.expm1(q) - q)) * on).sum() * s["scale"]
            d = torch.where(shut, 0.0, -a * r) - s["kl"] * torch.expm1(q)
        d = d * on * s["scale"]
        grad[t] = -torch.exp(lp) * d
        grad[t][row, cols] += d
    if op == "token_logp":
        return logp
    return {"loss": loss.reshape(1), "logp": logp, "dlogits": grad}
