"""fp64 CPU oracle of the language-model operators (include/lstmss.h): the
embedding lookup and its gradient, dropout with a computed mask, and the
vocabulary losses.  Plain numpy, one formula at a time; it shares no code with
the GPU path."""
from __future__ import annotations

import numpy as np

M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85
LOW = 0xFFFFFFFF


def philox(counter: int, seed: int, high: int = 0):
    """Philox4x32-10: four 32-bit words of the 128-bit counter whose low 64 bits
    are `counter` and whose high 64 bits are `high`."""
    c = [counter & LOW, (counter >> 32) & LOW, high & LOW, (high >> 32) & LOW]
    k0, k1 = seed & LOW, (seed >> 32) & LOW
    for _ in range(10):
        a, b = M0 * c[0], M1 * c[2]
        c = [(b >> 32) ^ c[1] ^ k0, b & LOW, (a >> 32) ^ c[3] ^ k1, a & LOW]
        k0, k1 = (k0 + W0) & LOW, (k1 + W1) & LOW
    return c


def threshold(p: float) -> int:
    return min(int(np.rint(float(np.float32(p)) * 65536.0)), 65535)


def keep_at(elements, p, seed, offset=0, period=0):
    """Which of the given element indices are kept (python integers)."""
    thr, out = threshold(p), []
    words = {}
    for e in elements:
        g = offset + (int(e) % period if period else int(e))
        c = (g // 8) % 2**64
        if c not in words:
            words[c] = philox(c, seed)
        k = g % 8
        out.append(((words[c][k // 2] >> (16 * (k % 2))) & 0xFFFF) >= thr)
    return np.array(out, bool)


def keep(n, p, seed, offset=0, period=0):
    """keep_at of 0 .. n-1 (vectorised over counters)."""
    m = min(n, period) if period else n
    u = np.uint64
    at = (np.arange(-(-m // 8), dtype=np.uint64) + u(offset // 8))
    c = [at & u(LOW), at >> u(32), np.zeros_like(at), np.zeros_like(at)]
    k0, k1 = seed & LOW, (seed >> 32) & LOW
    for _ in range(10):
        a, b = u(M0) * c[0], u(M1) * c[2]
        c = [(b >> u(32)) ^ c[1] ^ u(k0), b & u(LOW), (a >> u(32)) ^ c[3] ^ u(k1), a & u(LOW)]
        k0, k1 = (k0 + W0) & LOW, (k1 + W1) & LOW
    half = [h for w in c for h in (w & u(0xFFFF), w >> u(16))]
    bits = np.stack(half, 1).reshape(-1)[:m]
    mask = bits >= threshold(p)
    return np.resize(mask, n) if period else mask


def keep_scale(p) -> float:
    return 65536.0 / (65536.0 - threshold(p))


def dropout(x, p, seed, offset=0, period=0):
    x = np.asarray(x, np.float64)
    mask = keep(x.size, p, seed, offset, period).reshape(x.shape)
    return np.where(mask, x, 0.0) * np.where(mask, keep_scale(p), 0.0)


def embed(tokens, E, scale=1.0):
    """x [T][I][B]."""
    tokens, E = np.asarray(tokens), np.asarray(E, np.float64)
    x = np.zeros((tokens.shape[0], E.shape[1], tokens.shape[1]))
    for t in range(tokens.shape[0]):
        for b in range(tokens.shape[1]):
            if 0 <= tokens[t, b] < E.shape[0]:
                x[t, :, b] = scale * E[tokens[t, b]]
    return x


def embed_grad(tokens, dX, V, scale=1.0):
    """(dE [V][I], how many positions each row sums [V], sum of the terms' sizes [V][I])."""
    tokens, dX = np.asarray(tokens), np.asarray(dX, np.float64)
    dE, size = np.zeros((V, dX.shape[1])), np.zeros((V, dX.shape[1]))
    count = np.zeros(V, np.int64)
    for t in range(tokens.shape[0]):
        for b in range(tokens.shape[1]):
            v = tokens[t, b]
            if 0 <= v < V:
                dE[v] += scale * dX[t, :, b]
                size[v] += np.abs(scale * dX[t, :, b])
                count[v] += 1
    return dE, count, size


def log_softmax(logits):
    """Over the middle axis of [T][V][B]."""
    x = np.asarray(logits, np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        m = x.max(1, keepdims=True)
        z = x - np.where(np.isneginf(m), 0.0, m)
        return z - np.log(np.exp(z).sum(1, keepdims=True))


def _parts(logits, targets, weights):
    T, V, B = np.shape(logits)
    targets = np.asarray(targets)
    w = np.ones((T, B)) if weights is None else np.asarray(weights, np.float64)
    on = (targets >= 0) & (targets < V) & (w != 0)
    lsm = log_softmax(logits)
    logp = np.zeros((T, B))
    for t, b in zip(*np.nonzero(on)):
        logp[t, b] = lsm[t, targets[t, b], b]
    return targets, w, on, lsm, logp


def _grad(lsm, targets, on, g):
    d = np.zeros(lsm.shape)
    for t, b in zip(*np.nonzero(on & (g != 0))):
        d[t, :, b] = -g[t, b] * np.exp(lsm[t, :, b])
        d[t, targets[t, b], b] += g[t, b]
    return d


def token_logp(logits, targets):
    return _parts(logits, targets, None)[4]


def xent(logits, targets, weights=None, scale=1.0):
    """(loss, logp, dL/dlogp [T][B], dlogits)."""
    targets, w, on, lsm, logp = _parts(logits, targets, weights)
    g = np.where(on, -scale * w, 0.0)
    return float((g[on] * logp[on]).sum()), logp, g, _grad(lsm, targets, on, g)


def policy_loss(logits, targets, old, ref, adv, weights=None, clip_low=0.2, clip_high=0.2, kl=0.0,
                scale=1.0):
    """(loss, logp, dL/dlogp [T][B], dlogits); old / ref may be None."""
    targets, w, on, lsm, logp = _parts(logits, targets, weights)
    loss, g = 0.0, np.zeros(logp.shape)
    for t, b in zip(*np.nonzero(on)):
        lp, A = logp[t, b], float(adv[t][b])
        r = 1.0 if old is None else np.exp(lp - float(old[t][b]))
        c = min(max(r, 1.0 - float(np.float32(clip_low))), 1.0 + float(np.float32(clip_high)))
        term, dg = (-r * A, -r * A) if r * A <= c * A else (-c * A, 0.0)
        if kl:
            q = float(ref[t][b]) - lp
            term += kl * (np.expm1(q) - q)
            dg -= kl * np.expm1(q)
        loss += scale * w[t, b] * term
        g[t, b] = scale * w[t, b] * dg
    return loss, logp, g, _grad(lsm, targets, on, g)
