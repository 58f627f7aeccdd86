"""GPU parity of the language-model operators against the fp64 oracle
(oracle/language.py).

Bounds, u = 2^-24:
  embed, dropout   bit for bit: one product or two in fp32, one rounding
  embed_grad       row of n positions: n sums and two products in fp32, so
                   (n + 3) u times the sum of the terms' sizes
  logp             a sum of V exponentials, each within 8 u (the argument's
                   product and the exponential) and of either sign: 16 sqrt(V) u
                   for the sum's logarithm, one more rounding of logp itself;
                   small V: 16 u
  dlogits          g * softmax: the exponential's argument z within |z| u three
                   times over, the sum as above, four products
  loss             sum of the terms' derivative times logp's bound, one rounding
A bf16 output adds 2^-8 of its size (half an ulp, and the fp32 value's share)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import language as O

pytestmark = pytest.mark.gpu
U = 2.0**-24
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1806_00512_amd.lstmss as lstmss
    lstmss.load()
    return lstmss


def up(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


def np64(t):
    return t.detach().double().cpu().numpy()


def tokens_of(rng, T, B, V, kind):
    if kind == "pad":
        return np.full((T, B), -1, np.int32)
    if kind == "one":
        return np.full((T, B), V - 1, np.int32)
    if kind == "zipf":
        return (float(V) ** rng.random((T, B)) - 1.0).astype(np.int32).clip(0, V - 1)
    tok = rng.integers(0, V, (T, B)).astype(np.int32)
    bad = rng.random((T, B)) < 0.2
    return np.where(bad, rng.choice(np.array([-1, V, -2**31, 2**31 - 1], np.int32), (T, B)), tok)


def odd_start(shape, dtype, skip):
    """A contiguous tensor whose first element is `skip` elements off a 256-byte boundary,
    between guard values."""
    n = int(np.prod(shape))
    whole = torch.full((n + 128,), 7.0, dtype=dtype, device=DEV)
    return whole, whole[skip:skip + n].view(shape)


def guards_hold(whole, skip, n):
    assert (whole[:skip] == 7).all() and (whole[skip + n:] == 7).all()


# ------------------------------------------------------------ dropout

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,p,offset,period,skip", [
    (1, 0.5, 0, 0, 0), (7, 0.5, 8, 0, 0), (8, 0.1, 0, 0, 0), (9, 0.9, 2**63, 0, 0),
    (100003, 0.3, 0, 0, 0), (65536, 0.5, 2**64 - 64, 0, 0), (4096, 0.25, 0, 0, 1),
    (5003, 0.65, 24, 0, 3), (4096, 0.5, 0, 1, 0), (5000, 0.5, 0, 7, 0), (4096, 0.5, 0, 64, 0),
    (40961, 0.4, 16, 1000, 0), (3000, 0.5, 0, 8, 2), (4100, 0.5, 0, 4096, 0),
    (300, 0.5, 0, 1 << 50, 0), (1000, 0.0, 0, 0, 0), (1000, 0.99999, 0, 0, 0),
    (600000, 0.5, 0, 200, 0), (600000, 0.5, 8, 40000, 0)])
def test_dropout(L, dtype, n, p, offset, period, skip):
    rng = np.random.default_rng(n)
    seed = 0xFEDCBA9876543210 ^ n
    x = rng.standard_normal(n).astype(np.float32)
    x[rng.integers(0, n, 1 + n // 50)] = np.nan
    x[rng.integers(0, n, 1 + n // 50)] = np.inf
    whole, xt = odd_start((n,), TYPES[dtype], skip)
    xt.copy_(up(x, TYPES[dtype]))
    outw, out = odd_start((n,), TYPES[dtype], skip)
    drop = L.drop(p, seed, offset % 2**64, period)
    L.dropout(xt, drop, out=out)
    guards_hold(outw, skip, n)
    # one product in fp32, rounded once to the storage type; a kept NaN stays one
    k = up(O.keep(n, p, seed, offset, period), torch.bool)
    scale = torch.tensor(O.keep_scale(p), dtype=torch.float32, device=DEV)
    ref = torch.where(k, xt.float() * scale, torch.zeros((), device=DEV)).to(TYPES[dtype])
    assert torch.equal(out.isnan(), ref.isnan())
    assert torch.equal(out.nan_to_num(nan=0.0), ref.nan_to_num(nan=0.0))
    assert (out[~k] == 0).all() and not torch.signbit(out[~k].float()).any()
    L.dropout(xt, drop, out=xt)     # in place: the same bits
    assert torch.equal(xt.nan_to_num(nan=5.0), out.nan_to_num(nan=5.0))
    guards_hold(whole, skip, n)


def test_dropout_mask_is_the_types_and_the_gradients(L):
    x = torch.ones(35, 650, 20, device=DEV)
    d = L.drop(0.5, 3, 8, 650 * 20)
    y, z = L.dropout(x, d), L.dropout(x.bfloat16(), d)
    assert torch.equal(y, z.float())
    assert torch.equal(y[0], y[34])
    # linear: the call on a gradient is the derivative of the call
    g = torch.randn_like(x)
    assert torch.equal(L.dropout(g, d), g * y)


def test_dropout_past_32_bits(L):
    n = 2**31 + 40
    x = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    L.dropout(x, L.drop(0.5, 11), out=x)
    for e0 in (0, 2**31 - 20, n - 20):
        at = list(range(e0, e0 + 20))
        assert torch.equal(x[e0:e0 + 20].cpu() != 0, torch.from_numpy(O.keep_at(at, 0.5, 11)))


# ------------------------------------------------------------ embedding

EMBED = [  # T, B, I, V, tokens
    (1, 1, 1, 1, "one"), (1, 1, 650, 100, "some"), (3, 5, 7, 11, "some"), (2, 64, 64, 50, "zipf"),
    (4, 33, 65, 40, "some"), (2, 128, 128, 1000, "zipf"), (1, 300, 130, 77, "some"),
    (5, 20, 650, 300, "zipf"), (3, 256, 96, 20, "zipf"), (2, 7, 1023, 9, "some"),
    (6, 16, 40, 30, "pad"), (9, 8, 24, 5, "one"), (1, 3, 4096, 64, "some"), (70, 1, 33, 12, "zipf"),
    (2, 1000, 6, 90, "some"), (2, 12, 64, 30, "some"), (1, 2048, 3, 5, "zipf")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,I,V,kind", EMBED)
@pytest.mark.parametrize("p,period,skip", [(0.0, 0, 0), (0.3, 0, 1), (0.5, 1, 0)])
def test_embed(L, dtype, T, B, I, V, kind, p, period, skip):
    rng = np.random.default_rng(T * B + I)
    tok = tokens_of(rng, T, B, V, kind)
    E = up(rng.standard_normal((V, I)).astype(np.float32), TYPES[dtype])
    if skip:
        _, Es = odd_start((V, I), TYPES[dtype], skip)
        E = Es.copy_(E)
    scale = np.float32(1.7)
    drop = L.drop(p, 99, 16, period * I * B) if p else None
    whole, out = odd_start((T, I, B), TYPES[dtype], skip)
    L.embed(up(tok, torch.int32), E, scale=float(scale), drop=drop, out=out)
    guards_hold(whole, skip, T * I * B)
    # the products in fp32 as the operator forms them, rounded once
    x = np.zeros((T, I, B), np.float32)
    Eh = E.float().cpu().numpy()
    for t in range(T):
        ok = (tok[t] >= 0) & (tok[t] < V)
        x[t][:, ok] = (Eh[tok[t, ok]] * scale).T
    if p:
        k = O.keep(x.size, p, 99, 16, period * I * B).reshape(x.shape)
        x = np.where(k, x * np.float32(O.keep_scale(p)), np.float32(0))
    assert torch.equal(out, up(x, TYPES[dtype]))
    assert np.abs(x - (O.embed(tok, Eh, float(scale)) if not p else
                       O.dropout(O.embed(tok, Eh, float(scale)), p, 99, 16, period * I * B))).max() < 1e-5


def test_embed_skips_rows_that_are_not_used(L):
    E = torch.full((4, 100), float("nan"), device=DEV)
    E[2] = 1.0
    tok = torch.tensor([[2, -1, 4, 2, 2**31 - 1]], dtype=torch.int32, device=DEV)
    x = L.embed(tok, E)
    assert torch.equal(x, torch.tensor([1.0, 0, 0, 1, 0], device=DEV).expand(1, 100, 5))


@pytest.mark.parametrize("T,B,I,V,kind", EMBED + [(64, 64, 40, 8, "zipf"), (100, 100, 12, 4000, "zipf"),
                                                  (40, 128, 30, 50, "one"), (33, 31, 200, 3, "some"),
                                                  (300, 100, 5, 20000, "zipf"), (128, 512, 3, 700, "some")])
@pytest.mark.parametrize("p,accumulate,skip", [(0.0, False, 0), (0.25, True, 0), (0.0, False, 1),
                                               (0.5, False, 3)])
def test_embed_grad(L, T, B, I, V, kind, p, accumulate, skip):
    rng = np.random.default_rng(T * B + I)
    tok = tokens_of(rng, T, B, V, kind)
    g = rng.standard_normal((T, I, B)).astype(np.float32)
    # what stands at padding takes no part, whatever it is
    padded = (tok < 0) | (tok >= V)
    g.transpose(0, 2, 1)[padded] = np.nan
    _, gt = odd_start((T, I, B), torch.float32, skip)
    gt.copy_(up(g))
    period = (I * B) if p == 0.5 else 0
    drop = L.drop(p, 5, 8, period) if p else None
    base = rng.standard_normal((V, I)).astype(np.float32) if accumulate else np.zeros((V, I), np.float32)
    whole, dE = odd_start((V, I), torch.float32, skip)
    dE.copy_(up(base)) if accumulate else dE.fill_(float("nan"))
    L.embed_grad(up(tok, torch.int32), gt, V, scale=1.3, drop=drop, accumulate=accumulate, dE=dE)
    guards_hold(whole, skip, V * I)
    first = dE.clone()
    gz = np.where(np.isnan(g), 0.0, g)
    if p:
        gz = O.dropout(gz, p, 5, 8, period)
    ref, count, size = O.embed_grad(tok, gz, V, float(np.float32(1.3)))
    tol = (count[:, None] + 3) * U * size + (U * np.abs(ref + base) if accumulate else 0)
    assert (np.abs(np64(dE) - (ref + base)) <= tol).all()
    absent = count == 0
    assert np.array_equal(dE.cpu().numpy()[absent], base[absent])
    # the order is the tokens': again, and on another workspace, the same bits
    dE.copy_(up(base))
    L.embed_grad(up(tok, torch.int32), gt, V, scale=1.3, drop=drop, accumulate=accumulate, dE=dE,
                 ws=torch.full((L.embed_grad_workspace_bytes(T, B, I, V) + 64,), 255, dtype=torch.uint8,
                               device=DEV))
    assert torch.equal(dE, first)


@pytest.mark.parametrize("T,B,I", [(3, 64, 70), (40, 64, 66), (2, 20, 30), (33, 100, 12)])
@pytest.mark.parametrize("period", [1, 13, 100, 1000003])
def test_masks_that_repeat_after_any_length(L, T, B, I, period):
    """Lookup and gradient with masks that repeat after no multiple of eight, few positions and many."""
    rng = np.random.default_rng(period)
    V = 40
    tok = tokens_of(rng, T, B, V, "some")
    E = rng.standard_normal((V, I)).astype(np.float32)
    g = rng.standard_normal((T, I, B)).astype(np.float32)
    drop = L.drop(0.4, 21, 16, period)
    x = L.embed(up(tok, torch.int32), up(E), drop=drop)
    k = O.keep(x.numel(), 0.4, 21, 16, period).reshape(T, I, B)
    ref = np.where(k, O.embed(tok, E).astype(np.float32) * np.float32(O.keep_scale(0.4)), np.float32(0))
    assert torch.equal(x, up(ref))
    dE = L.embed_grad(up(tok, torch.int32), up(g), V, drop=drop)
    want, count, size = O.embed_grad(tok, O.dropout(g, 0.4, 21, 16, period), V)
    assert (np.abs(np64(dE) - want) <= (count[:, None] + 3) * U * size).all()


def test_embed_grad_against_differences(L):
    """<G, embed(E)> differs between E + h and E - h by 2 h <G, embed'>: linear, so any h."""
    rng = np.random.default_rng(3)
    tok = up(tokens_of(rng, 5, 6, 8, "some"), torch.int32)
    G = up(rng.standard_normal((5, 10, 6)).astype(np.float32))
    E = up(rng.standard_normal((8, 10)).astype(np.float32))
    drop = L.drop(0.4, 1)
    dE = L.embed_grad(tok, G, 8, scale=2.0, drop=drop)
    H = up(rng.standard_normal((8, 10)).astype(np.float32))
    f = lambda e: (L.embed(tok, e, scale=2.0, drop=drop).double() * G.double()).sum()  # noqa: E731
    diff = (f(E + H) - f(E - H)) / 2
    # 30 x 10 products of size about 7, each within 4 u
    assert abs(float(diff - (dE.double() * H.double()).sum())) < 300 * 40 * 4 * U


# ------------------------------------------------------------ losses

LOSS = [  # T, V, B
    (1, 1, 1), (1, 2, 1), (1, 1000, 1), (2, 7, 3), (3, 100, 20), (1, 503, 33), (2, 64, 64),
    (2, 513, 130), (1, 300, 1000), (4, 3001, 8), (2, 10000, 16), (1, 97, 251), (3, 50, 24),
    (5, 257, 12), (1, 40, 2056), (1, 9001, 5), (2, 33, 4104), (1, 12, 3001), (9, 700, 17)]


def logits_of(rng, T, V, B, kind):
    x = rng.standard_normal((T, V, B)) * 3
    if kind == "wide":
        x *= 20
    if kind == "holes":         # words masked out of the vocabulary
        x[rng.random(x.shape) < 0.3] = -np.inf
        x[rng.random(x.shape) < 0.1] = np.finfo(np.float32).min
        x[:, 0] = 0.0           # (one word of every column stays)
    if kind == "far":           # a large common offset: only differences count
        x = x + 20000.0
    return x


def loss_inputs(T, V, B, kind, dtype, seed):
    rng = np.random.default_rng(seed)
    x = up(logits_of(rng, T, V, B, kind).astype(np.float32), TYPES[dtype])
    y = rng.integers(0, V, (T, B)).astype(np.int32)
    if kind == "holes":
        y[:] = np.where(rng.random((T, B)) < 0.5, 0, y)
    if kind in ("pad", "holes"):
        y = np.where(rng.random((T, B)) < 0.3, rng.choice(np.array([-1, V, -2**31, 2**31 - 1], np.int32), (T, B)), y)
    w = (rng.uniform(0.2, 2, (T, B)) * (rng.random((T, B)) < 0.8)).astype(np.float32)
    return rng, x, y, w


def logp_tol(V, logp):
    return U * (16 * np.sqrt(V) + 16 + 2 * np.abs(logp))


def check_grad(L, out, x, d, g, V, dtype, tol_lp, g_tol):
    """dlogits against the oracle's; g, g_tol [T][B]: dL/dlogp and its bound."""
    lsm = O.log_softmax(np64(x))
    p = np.exp(np.where(np.isnan(lsm), -np.inf, lsm))
    z = np.where(np.isfinite(lsm), np.abs(lsm), 0.0)
    lim = np.abs(g)[:, None] * p * (tol_lp[:, None] + (3 * z + 16) * U) + g_tol[:, None] * (1 + p)
    lim = lim + np.abs(d) * (2.0**-8 if dtype == "bf16" else 2 * U) + 2.0**-133
    err = np.abs(np64(out) - d)
    assert (err <= lim).all(), float((err - lim).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "pad", "holes", "wide", "far"])
@pytest.mark.parametrize("T,V,B", LOSS)
def test_xent(L, dtype, kind, T, V, B):
    rng, x, y, w = loss_inputs(T, V, B, kind, dtype, T + V * 7 + B)
    out = L.xent(x, up(y, torch.int32), weights=up(w), scale=0.25)
    loss, logp, g, d = O.xent(np64(x), y, w, 0.25)
    tol = logp_tol(V, np.where(np.isfinite(logp), logp, 0))
    got = np64(out["logp"])
    assert np.array_equal(np.isneginf(got), np.isneginf(logp))
    fin = np.isfinite(logp)
    assert (np.abs(got[fin] - logp[fin]) <= tol[fin]).all()
    if np.isfinite(loss):
        assert abs(float(out["loss"]) - loss) <= (np.abs(g) * tol).sum() + 2 * U * (abs(loss) + np.abs(g * np.where(fin, logp, 0)).sum())
    else:
        assert np.isposinf(float(out["loss"]))
    check_grad(L, out["dlogits"], x, d, g, V, dtype, tol, 2 * U * np.abs(g))
    off = (y < 0) | (y >= V) | (w == 0)
    assert (np64(out["dlogits"]).transpose(0, 2, 1)[off] == 0).all() and (got[off] == 0).all()
    # the targets' logp alone; without weights; in place
    lone = np64(L.token_logp(x, up(y, torch.int32)))
    ref = O.token_logp(np64(x), y)
    fin = np.isfinite(ref)
    assert (np.abs(lone[fin] - ref[fin]) <= logp_tol(V, ref[fin])).all()
    first = out["dlogits"].clone()
    again = L.xent(x, up(y, torch.int32), weights=up(w), scale=0.25, out={"dlogits": x})
    assert torch.equal(x, first) and torch.equal(again["logp"], out["logp"]) and torch.equal(again["loss"], out["loss"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mode", ["all", "no_old", "no_ref", "no_weights"])
@pytest.mark.parametrize("T,V,B", LOSS)
def test_policy_loss(L, dtype, mode, T, V, B):
    rng, x, y, w = loss_inputs(T, V, B, "pad", dtype, T + V * 7 + B)
    lp = O.token_logp(np64(x), y)
    r = rng.uniform(-0.5, 0.5, (T, B))
    lo, hi, kl = 0.2, 0.3, 0.0 if mode == "no_ref" else 0.1
    for c in (np.log(1 - lo), np.log(1 + hi)):   # off the corners by more than logp's bound
        r = np.where(np.abs(r - c) < 1e-2, c + 2e-2, r)
    old, ref = (lp - r).astype(np.float32), (lp + rng.standard_normal((T, B)) * 0.3).astype(np.float32)
    adv = rng.standard_normal((T, B)).astype(np.float32)
    a = {"old": None if mode == "no_old" else old, "ref": None if mode == "no_ref" else ref, "adv": adv,
         "weights": None if mode == "no_weights" else w}
    out = L.policy_loss(x, up(y, torch.int32), **{k: None if v is None else up(v) for k, v in a.items()},
                        clip_low=lo, clip_high=hi, kl=kl, scale=0.125)
    loss, logp, g, d = O.policy_loss(np64(x), y, a["old"], a["ref"], adv, a["weights"], lo, hi,
                                     float(np.float32(kl)), 0.125)
    tol = logp_tol(V, logp)
    assert (np.abs(np64(out["logp"]) - logp) <= tol).all()
    # dL/dlogp and the loss move with logp by w * scale * (|r adv| + kl e^q) at most
    w1 = np.ones((T, B)) if a["weights"] is None else w
    slope = 0.125 * w1 * (np.abs(adv) * np.exp(0.55) + kl * np.exp(np.abs(ref - lp) * (kl > 0)))
    slope = slope * ((y >= 0) & (y < V))
    assert abs(float(out["loss"]) - loss) <= (2 * slope * (tol + 4 * U)).sum() + U * abs(loss)
    check_grad(L, out["dlogits"], x, d, g, V, dtype, tol, slope * tol + 4 * U * np.abs(g))
    no = L.policy_loss(x, up(y, torch.int32), **{k: None if v is None else up(v) for k, v in a.items()},
                       clip_low=lo, clip_high=hi, kl=kl, scale=0.125, want_grad=False)
    assert "dlogits" not in no and torch.equal(no["loss"], out["loss"]) and torch.equal(no["logp"], out["logp"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,B", [(50, 6), (1000, 40), (333, 20)])
def test_padding_hides_anything(L, dtype, V, B):
    """Columns that take no part may hold NaN, infinities or nothing but -inf."""
    rng, x, y, w = loss_inputs(2, V, B, "plain", dtype, V)
    clean = L.xent(x, up(y, torch.int32), weights=up(w))
    y2 = y.copy()
    y2[0, 1], w[1, 2] = -1, 0.0
    for t, b in ((0, 1), (1, 2)):
        for value in (float("nan"), float("inf"), -float("inf")):
            x[t, ::2, b] = value
            x[t, 1::2, b] = -float("inf")
            out = L.xent(x, up(y2, torch.int32), weights=up(w))
            assert torch.isfinite(out["loss"]).all()
            assert (out["dlogits"][t, :, b] == 0).all() and float(out["logp"][t, b]) == 0
        x[t, :, b] = 0
    keep = [(t, b) for t in range(2) for b in range(B) if (t, b) not in ((0, 1), (1, 2))]
    for t, b in keep:
        assert torch.equal(out["dlogits"][t, :, b], clean["dlogits"][t, :, b])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_columns_without_a_value(L, dtype):
    """A column of -inf alone has no softmax: NaN, as the formula gives; so has one with +inf or NaN."""
    x = torch.zeros(1, 40, 5, dtype=TYPES[dtype], device=DEV)
    x[0, :, 1] = -float("inf")
    x[0, 7, 2] = float("inf")
    x[0, 39, 3] = float("nan")
    out = L.xent(x, torch.zeros(1, 5, dtype=torch.int32, device=DEV), scale=1.0)
    lp = out["logp"][0]
    assert torch.isnan(lp[1:4]).logical_or(torch.isneginf(lp[1:4])).all()
    assert torch.isnan(lp[1]) and torch.isnan(lp[3])
    assert torch.isnan(out["dlogits"][0, :, 1]).all() and torch.isnan(out["dlogits"][0, :, 3]).all()
    for b in (0, 4):
        assert abs(float(lp[b]) + np.log(40)) < 1e-5 and torch.isfinite(out["dlogits"][0, :, b]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,B,skip", [(2, 301, 20, 1), (1, 1000, 64, 3), (3, 77, 7, 5)])
def test_loss_alignment(L, dtype, T, V, B, skip):
    """Tensors that start anywhere give the same bits and write nothing outside."""
    rng, x, y, w = loss_inputs(T, V, B, "pad", dtype, 5)
    ref = L.xent(x, up(y, torch.int32), weights=up(w))
    _, xs = odd_start((T, V, B), TYPES[dtype], skip)
    xs.copy_(x)
    whole, ds = odd_start((T, V, B), TYPES[dtype], skip)
    lw, lp = odd_start((T, B), torch.float32, skip)
    out = L.xent(xs, up(y, torch.int32), weights=up(w), out={"dlogits": ds, "logp": lp})
    tol = logp_tol(V, np64(ref["logp"]))
    assert (np.abs(np64(lp) - np64(ref["logp"])) <= 2 * tol).all()
    close = torch.allclose(ds.float(), ref["dlogits"].float(), rtol=2.0**-7 if dtype == "bf16" else 1e-4, atol=1e-9)
    assert close
    guards_hold(whole, skip, T * V * B)
    guards_hold(lw, skip, T * B)


# T, V, B whose sums are taken by each of the kernels in both types: one launch for sums and
# terms; whole rows to a work-group; windows of long rows
OFFSET_SHAPES = [(3, 97, 20), (2, 5003, 33), (1, 20000, 8), (1, 700, 2056), (1, 1300, 1031)]


def offset_logits(rng, T, V, B, dtype):
    """Columns around offsets of every size, and columns that hold one finite value alone (a
    vocabulary masked out as a whole), as they are stored."""
    most = torch.finfo(TYPES[dtype]).max
    spread = [0.0, 1e5, -1e6, 4e6, -1e7, 1e9, -1e9, 1e20]
    alone = [-1e9, -most, most, 1e9, -1e4, 0.0]
    x = up(rng.standard_normal((T, V, B)).astype(np.float32) * 3).double()
    for b in range(B):
        k = b % (len(spread) + len(alone))
        if k < len(spread):
            x[:, :, b] += spread[k]
        else:
            x[:, :, b] = alone[k - len(spread)]
    return x.to(TYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,B", OFFSET_SHAPES)
def test_gradients_at_any_offset(L, dtype, T, V, B):
    """What is common to a column takes no part, however large: the bounds are those of logits
    around zero.  A column of one value alone has the uniform distribution's gradient."""
    rng = np.random.default_rng(V)
    x = offset_logits(rng, T, V, B, dtype)
    y = rng.integers(0, V, (T, B)).astype(np.int32)
    w = rng.uniform(0.2, 2, (T, B)).astype(np.float32)
    yt = up(y, torch.int32)
    loss, logp, g, d = O.xent(np64(x), y, w, 0.25)
    out = L.xent(x, yt, weights=up(w), scale=0.25)
    tol = logp_tol(V, logp)
    assert (np.abs(np64(out["logp"]) - logp) <= tol).all()
    assert abs(float(out["loss"]) - loss) <= (np.abs(g) * tol).sum() + 2 * U * (abs(loss) + np.abs(g * logp).sum())
    check_grad(L, out["dlogits"], x, d, g, V, dtype, tol, 2 * U * np.abs(g))
    # the policy loss, unclipped: r is within [1 - 2^-4, 1 + 2^-4]
    old = (logp + rng.uniform(-0.06, 0.06, (T, B))).astype(np.float32)
    ref = (logp + rng.uniform(-0.3, 0.3, (T, B))).astype(np.float32)
    adv = rng.standard_normal((T, B)).astype(np.float32)
    out = L.policy_loss(x, yt, up(old), up(ref), up(adv), weights=up(w), kl=0.125, scale=0.25)
    _, _, g, d = O.policy_loss(np64(x), y, old, ref, adv, w, 0.2, 0.2, 0.125, 0.25)
    slope = 0.25 * w * (np.abs(adv) * np.exp(0.07) + 0.125 * np.exp(0.31))
    check_grad(L, out["dlogits"], x, d, g, V, dtype, tol, slope * tol + 4 * U * np.abs(g))


def test_xent_against_differences(L):
    """Central differences of the loss along one direction: h^2 / 6 of its third derivative and
    the loss's rounding over h."""
    rng, x, y, w = loss_inputs(2, 50, 6, "pad", "f32", 9)
    wt, yt = up(w), up(y, torch.int32)
    d = L.xent(x, yt, weights=wt, scale=1.0)["dlogits"]
    v = up(rng.standard_normal((2, 50, 6)).astype(np.float32))
    h = 1e-2
    f = [float(L.xent(x + s * h * v, yt, weights=wt, scale=1.0, want_grad=False)["loss"]) for s in (1, -1)]
    size = float(w.sum())
    assert abs((f[0] - f[1]) / (2 * h) - float((d.double() * v.double()).sum())) < \
        size * (h * h * 30 / 6 + 200 * U / h)


def test_loss_past_32_bits(L):
    T, V, B = 17, 32000, 4096     # 2.2e9 logits
    x = torch.empty((T, V, B), dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    for t in range(T):
        x[t] = torch.randn((V, B), generator=g, device=DEV).bfloat16()
    y = torch.randint(0, V, (T, B), generator=g, device=DEV, dtype=torch.int32)
    cols = [0, 1, 4095]
    keep = {(t, b): x[t, :, b].clone() for t in (0, 8, 16) for b in cols}
    out = L.xent(x, y, scale=1.0, out={"dlogits": x})
    for (t, b), c in keep.items():
        lsm = torch.log_softmax(c.double().cpu(), 0)
        v = int(y[t, b])
        assert abs(float(out["logp"][t, b]) - float(lsm[v])) <= logp_tol(V, float(lsm[v]))
        d = torch.exp(lsm)
        d[v] -= 1
        assert torch.allclose(x[t, :, b].double().cpu(), d, rtol=2.0**-7, atol=0)


# ------------------------------------------------------------ large tensors

@pytest.mark.parametrize("dtype,n,period", [("f32", 9000000, 0), ("bf16", 17000003, 0), ("f32", 8500001, 4096),
                                            ("bf16", 17000000, 1000003)])
def test_dropout_of_large_tensors(L, dtype, n, period):
    """32 MB and more are written another way."""
    x = torch.randn(n, device=DEV).to(TYPES[dtype])
    y = L.dropout(x, L.drop(0.3, 17, 8, period))
    k = up(O.keep(n, 0.3, 17, 8, period), torch.bool)
    scale = torch.tensor(O.keep_scale(0.3), dtype=torch.float32, device=DEV)
    assert torch.equal(y, torch.where(k, x.float() * scale, torch.zeros((), device=DEV)).to(TYPES[dtype]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,I,p", [(40, 128, 2048, 0.2), (40, 128, 2048, 0.0), (45, 100, 2047, 0.2),
                                     (9000, 1, 2048, 0.0), (1300, 13, 1030, 0.2)])
def test_embed_of_large_tensors(L, dtype, T, B, I, p):
    rng = np.random.default_rng(T)
    tok = up(tokens_of(rng, T, B, 500, "some"), torch.int32)
    E = torch.randn((500, I), device=DEV).to(TYPES[dtype])
    x = L.embed(tok, E, scale=0.7, drop=L.drop(p, 3) if p else None)
    ok = (tok >= 0) & (tok < 500)
    rows = E[torch.where(ok, tok, 0).long()].float() * torch.tensor(0.7, device=DEV)
    ref = torch.where(ok[..., None], rows, torch.zeros((), device=DEV)).permute(0, 2, 1)
    if p:
        k = up(O.keep(x.numel(), p, 3).reshape(x.shape), torch.bool)
        ref = torch.where(k, ref * torch.tensor(O.keep_scale(p), dtype=torch.float32, device=DEV), torch.zeros((), device=DEV))
    assert torch.equal(x, ref.to(TYPES[dtype]))


@pytest.mark.parametrize("T,B,I,V,p", [(50, 128, 2048, 4000, 0.0), (50, 128, 2048, 4000, 0.3), (60, 64, 1500, 900, 0.0),
                                       (16, 96, 1100, 500, 0.2), (1, 1900, 2100, 300, 0.0), (70, 30, 1020, 40, 0.0),
                                       (100, 2048, 8, 1000000, 0.0), (2, 40000, 16, 5, 0.3), (40000, 1, 33, 70, 0.0),
                                       (1, 1, 30000, 1000, 0.5)])
def test_embed_grad_of_large_tensors(L, T, B, I, V, p):
    rng = np.random.default_rng(I)
    tok = up(tokens_of(rng, T, B, V, "zipf"), torch.int32)
    g = torch.randn((T, I, B), device=DEV)
    dE = L.embed_grad(tok, g, V, scale=1.5, drop=L.drop(p, 2) if p else None)
    d = g.double()
    if p:
        d = d * up(O.keep(g.numel(), p, 2).reshape(g.shape), torch.float64) * O.keep_scale(p)
    rows = d.permute(0, 2, 1).reshape(T * B, I) * 1.5
    at = tok.reshape(-1).long()
    ref = torch.zeros((V, I), dtype=torch.float64, device=DEV).index_add_(0, at, rows)
    size = torch.zeros((V, I), dtype=torch.float64, device=DEV).index_add_(0, at, rows.abs())
    count = torch.bincount(at, minlength=V).double()
    assert ((dE.double() - ref).abs() <= (count[:, None] + 3) * U * size + 1e-13 * size).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,B", [(2, 20000, 250), (3, 9999, 333), (2, 30000, 640), (4, 40000, 500), (1, 30011, 2100),
                                   (31, 32001, 128), (33, 17001, 3), (5, 16411, 20), (1, 20001, 1), (2, 17003, 130),
                                   (40, 4999, 33), (100, 2000, 33), (12, 16500, 7), (1, 17000, 2100), (2, 50, 9000),
                                   (3, 20000, 1031), (300, 1000, 9), (1, 17001, 256), (7, 16400, 255)])
@pytest.mark.parametrize("skip", [(0, 0), (1, 1), (3, 6)])
def test_xent_of_large_tensors(L, dtype, T, V, B, skip):
    """Small logits take one kernel for sums and terms, larger ones two; from 32 MB on the gradient
    is written another way, from 224 MB on part of the logits is read another way: against the same
    formula in fp64, step by step, with tensors that start anywhere."""
    g = torch.Generator(device=DEV)
    g.manual_seed(V)
    whole, x = odd_start((T, V, B), TYPES[dtype], skip[0])
    x.copy_(torch.randn((T, V, B), generator=g, device=DEV) * 3)
    y = torch.randint(-1, V, (T, B), generator=g, device=DEV, dtype=torch.int32)
    whole, d = odd_start((T, V, B), TYPES[dtype], skip[1])
    out = L.xent(x, y, scale=0.5, out={"dlogits": d})
    guards_hold(whole, skip[1], d.numel())
    assert abs(float(out["loss"]) + 0.5 * float(out["logp"].double().sum())) <= 4 * U * 0.5 * float(out["logp"].double().abs().sum())
    for t in range(T):
        lsm = torch.log_softmax(x[t].double(), 0)
        on = (y[t] >= 0).double()
        at = y[t].clamp(min=0).long()
        lp = lsm.gather(0, at[None])[0] * on
        tol = U * (16 * np.sqrt(V) + 16 + 2 * lp.abs())
        assert ((out["logp"][t].double() - lp).abs() <= tol).all()
        p = lsm.exp()
        ref = 0.5 * on * p
        ref[at, torch.arange(B, device=DEV)] -= 0.5 * on
        lim = 0.5 * on * p * (tol + (3 * lsm.abs() + 16) * U) + 2 * U * 0.5 + ref.abs() * (2.0**-8 if dtype == "bf16" else 2 * U) + 2.0**-133
        assert ((d[t].double() - ref).abs() <= lim).all()


# ------------------------------------------------------------ calls

def test_long_rows_as_one_step(L):
    """[1][V][T * B] is the same loss as [T][V][B]: the layout of one product for all steps."""
    rng, x, y, w = loss_inputs(6, 400, 96, "pad", "f32", 4)
    a = L.xent(x, up(y, torch.int32), weights=up(w), scale=1.0)
    flat = x.permute(1, 0, 2).reshape(1, 400, -1).contiguous()
    b = L.xent(flat, up(y, torch.int32).view(1, -1), weights=up(w).view(1, -1), scale=1.0)
    assert np.abs(np64(a["logp"]).reshape(-1) - np64(b["logp"]).reshape(-1)).max() <= 2 * logp_tol(400, 20.0)
    assert torch.allclose(a["dlogits"].permute(1, 0, 2).reshape(1, 400, -1), b["dlogits"], rtol=1e-4, atol=1e-9)


def every_call(L, s):
    """One call of every operator on the tensors of s (written to s's outputs)."""
    d = L.drop(0.5, 7)
    st = s.get("stream")
    L.embed(s["tok"], s["E"], drop=d, out=s["x"], stream=st)
    L.dropout(s["x"], d, out=s["y"], stream=st)
    L.embed_grad(s["tok"], s["y"], s["E"].shape[0], drop=d, dE=s["dE"], ws=s["ws1"], stream=st)
    L.xent(s["z"], s["tgt"], out=s["o1"], ws=s["ws2"], stream=st)
    L.policy_loss(s["z"], s["tgt"], s["o1"]["logp"], s["o1"]["logp"], s["adv"], kl=0.1, out=s["o2"], ws=s["ws2"],
                  stream=st)
    L.token_logp(s["z"], s["tgt"], logp=s["lp"], ws=s["ws2"], stream=st)


def call_state(L, seed, T=7, B=20, I=130, V=900):
    rng = np.random.default_rng(seed)
    s = {"tok": up(tokens_of(rng, T, B, V, "zipf"), torch.int32),
         "tgt": up(tokens_of(rng, T, B, V, "some"), torch.int32),
         "E": up(rng.standard_normal((V, I)).astype(np.float32)),
         "z": up(rng.standard_normal((T, V, B)).astype(np.float32)),
         "adv": up(rng.standard_normal((T, B)).astype(np.float32))}
    f = dict(dtype=torch.float32, device=DEV)
    s.update(x=torch.zeros((T, I, B), **f), y=torch.zeros((T, I, B), **f), dE=torch.zeros((V, I), **f),
             lp=torch.zeros((T, B), **f))
    for k in ("o1", "o2"):
        s[k] = {"loss": torch.zeros(1, **f), "logp": torch.zeros((T, B), **f), "dlogits": torch.zeros((T, V, B), **f)}
    s["ws1"] = torch.empty(L.embed_grad_workspace_bytes(T, B, I, V), dtype=torch.uint8, device=DEV)
    s["ws2"] = torch.empty(L.loss_workspace_bytes(T, B, V), dtype=torch.uint8, device=DEV)
    return s


def outputs(s):
    return [s["x"], s["y"], s["dE"], s["lp"]] + [s[k][n] for k in ("o1", "o2") for n in ("loss", "logp", "dlogits")]


def test_calls_on_another_stream(L):
    s = call_state(L, 1)
    every_call(L, s)
    ref = [t.clone() for t in outputs(s)]
    torch.cuda.synchronize()
    for t in outputs(s):
        t.fill_(float("nan"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s["stream"] = side
    every_call(L, s)
    # and with buffers of the call's own, freed while the stream still runs
    own = L.xent(s["z"], s["tgt"], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(outputs(s), ref))
    assert torch.equal(own["dlogits"], s["o1"]["dlogits"])


def test_new_tensors_of_a_call_on_another_stream(L):
    """They are not made of blocks that the current stream's work may still use."""
    d = L.drop(0.5, 7)
    x = torch.randn(3, 1000, 777, device=DEV)
    ref = L.dropout(x, d)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    freed = torch.empty_like(x)
    at = freed.data_ptr()
    del freed
    y = L.dropout(x, d, stream=side)
    side.synchronize()
    assert y.data_ptr() != at and torch.equal(y, ref)
    again = torch.empty_like(x)
    assert again.data_ptr() == at          # it is still the current stream's


def test_calls_in_a_captured_graph(L):
    """Recorded by the caller and replayed, with eager work between: every replay gives the
    eager call's bits."""
    s = call_state(L, 2)
    every_call(L, s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        every_call(L, s)
    for k in range(4):
        new = call_state(L, 10 + k)
        for n in ("tok", "tgt", "E", "z", "adv"):
            s[n].copy_(new[n])
        every_call(L, new)
        for t in outputs(s):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs(s), outputs(new))), k


def test_timing_hooks_see_the_calls(L):
    s = call_state(L, 3)
    L.timing_enable(True)
    try:
        L.timing_reset()
        every_call(L, s)
        ms, n = L.timing_read()["aux"]
        assert n == 6 and ms > 0
    finally:
        L.timing_enable(False)
        L.timing_reset()


def test_binding_refusals(L):
    s = call_state(L, 4)
    z, tgt, tok, E = s["z"], s["tgt"], s["tok"], s["E"]
    for bad in (lambda: L.embed(tok.long(), E), lambda: L.embed(tok.t(), E), lambda: L.embed(tok, E.half()),
                lambda: L.embed(tok, E[:, ::2]), lambda: L.embed(tok, E, out=s["x"][:-1]),
                lambda: L.embed(tok[0], E),
                lambda: L.embed_grad(tok, s["x"].bfloat16(), 900), lambda: L.embed_grad(tok, s["x"][:, :, :-1], 900),
                lambda: L.embed_grad(tok, s["x"], 900, accumulate=True), lambda: L.embed_grad(tok, s["x"], 900, dE=E.t()),
                lambda: L.xent(z, tgt.long()), lambda: L.xent(z, tgt[:-1]), lambda: L.xent(z.permute(0, 2, 1), tgt),
                lambda: L.xent(z[0], tgt), lambda: L.xent(z, tgt, weights=s["adv"].double()),
                lambda: L.xent(z, tgt, out={"dlogits": z.bfloat16()}), lambda: L.xent(z.half(), tgt),
                lambda: L.dropout(z[:, ::2], L.drop(0.5, 1)), lambda: L.dropout(z, L.drop(0.5, 1), out=z.bfloat16()),
                lambda: L.xent(z, tgt.cpu()), lambda: L.token_logp(z, tgt, logp=s["lp"].cpu())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: L.embed(tok, E, drop=0.5), lambda: L.dropout(z, None), lambda: L.dropout(z, 0.5),
                lambda: L.policy_loss(z, tgt, None, None, None) and None):
        with pytest.raises((TypeError, L.LstmssError)):
            bad()
    for bad in (lambda: L.dropout(z, L.drop(1.0, 1)), lambda: L.dropout(z, L.drop(0.5, 1, 4)),
                lambda: L.policy_loss(z, tgt, None, None, s["adv"], kl=0.1),
                lambda: L.policy_loss(z, tgt, None, None, s["adv"], clip_low=2.0),
                lambda: L.xent(z, tgt, scale=float("nan")),
                lambda: L.xent(z, tgt, ws=s["ws2"][:16]), lambda: L.dropout(z[:0], L.drop(0.5, 1))):
        with pytest.raises(L.LstmssError):
            bad()
    assert ctypes.sizeof(L.Drop) == 32 and ctypes.sizeof(L.Tokens) == 20
