"""CPU pins of the language-model oracle (oracle/language.py): the generator's
published known answer, the mask's rate and index rules, closed forms, and
gradients against central differences; and the refusals of the operators'
entry points, which run before anything touches a GPU."""
import ctypes

import numpy as np
import pytest

from oracle import language as O


@pytest.fixture(scope="module")
def L():
    import paper_1806_00512_amd.lstmss as lstmss
    lstmss.load()
    return lstmss


def test_philox_known_answer():
    # the published known answers of Philox4x32-10: counter and key all zero, all one
    assert O.philox(0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert O.philox(2**64 - 1, 2**64 - 1, 2**64 - 1) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


@pytest.mark.parametrize("n,p,offset,period", [(1, 0.5, 0, 0), (37, 0.1, 8, 0), (64, 0.9, 2**40, 0),
                                               (50, 0.3, 16, 7), (33, 0.5, 0, 100)])
def test_keep_matches_the_element_rule(n, p, offset, period):
    seed = 0x0123456789ABCDEF
    assert np.array_equal(O.keep(n, p, seed, offset, period),
                          O.keep_at(range(n), p, seed, offset, period))


@pytest.mark.parametrize("p", [0.1, 0.25, 0.5, 0.9])
def test_keep_rate(p):
    # n independent draws: the rate's deviation is sqrt(p (1 - p) / n), five of it allowed
    n = 1 << 18
    rate = 1.0 - O.keep(n, p, 12345).mean()
    assert abs(rate - O.threshold(p) / 65536.0) < 5 * np.sqrt(p * (1 - p) / n)


def test_keep_streams_differ_and_continue():
    a, b = O.keep(4096, 0.5, 1), O.keep(4096, 0.5, 2)
    assert 0.4 < (a == b).mean() < 0.6
    assert np.array_equal(O.keep(4096, 0.5, 1)[1024:], O.keep(3072, 0.5, 1, offset=1024))


def test_threshold_ends():
    assert O.threshold(0.0) == 0 and O.threshold(1e-6) == 0
    assert O.threshold(0.5) == 32768 and O.threshold(np.nextafter(np.float32(1), np.float32(0))) == 65535
    assert O.keep(100, 0.0, 3).all()


def test_dropout_masks_what_is_not_finite():
    x = np.array([np.nan, np.inf, -np.inf, 1.0] * 8)
    y = O.dropout(x, 0.5, 7)
    k = O.keep(32, 0.5, 7)
    assert (y[~k] == 0).all() and y[k & (x == 1)].tolist() == [2.0] * int((k & (x == 1)).sum())


def test_embed_grad_is_the_transpose():
    rng = np.random.default_rng(0)
    T, B, I, V = 4, 3, 5, 6
    tok = rng.integers(-1, V + 1, (T, B))
    E, G = rng.standard_normal((V, I)), rng.standard_normal((T, I, B))
    dE, count, _ = O.embed_grad(tok, G, V, 1.5)
    # <embed(E), G> = <E, embed_grad(G)>
    assert np.isclose((O.embed(tok, E, 1.5) * G).sum(), (E * dE).sum(), rtol=1e-12)
    assert count.sum() == ((tok >= 0) & (tok < V)).sum()


def differences(f, x, h=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        p, m = x.copy(), x.copy()
        p[i] += h
        m[i] -= h
        g[i] = (f(p) - f(m)) / (2 * h)
    return g


def policy_inputs(T, V, B, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((T, V, B)) * 2
    y = rng.integers(-1, V + 1, (T, B))
    lp = O.token_logp(x, y)
    r = rng.uniform(-0.4, 0.4, (T, B))
    for c in (np.log(0.8), np.log(1.3)):     # no ratio at a corner of the clip
        r = np.where(np.abs(r - c) < 1e-3, c + 1e-2, r)
    return x, y, lp - r, lp + rng.standard_normal((T, B)) * 0.3, rng.standard_normal((T, B)), \
        rng.uniform(0, 2, (T, B)) * (rng.random((T, B)) < 0.8)


def test_xent_gradient_against_differences():
    x, y, _, _, _, w = policy_inputs(3, 7, 4, 1)
    _, _, _, d = O.xent(x, y, w, 0.3)
    # central differences: h^2 / 6 of the third derivative (at most 1), and 1e-16 / h of rounding
    assert np.abs(d - differences(lambda z: O.xent(z, y, w, 0.3)[0], x)).max() < 1e-9


@pytest.mark.parametrize("kl", [0.0, 0.1])
def test_policy_gradient_against_differences(kl):
    x, y, old, ref, adv, w = policy_inputs(3, 7, 4, 2)
    f = lambda z: O.policy_loss(z, y, old, ref, adv, w, 0.2, 0.3, kl, 0.3)  # noqa: E731
    assert np.abs(f(x)[3] - differences(lambda z: f(z)[0], x)).max() < 1e-8


def test_policy_clips_one_side_only():
    x = np.zeros((1, 2, 4))
    lp = np.log(0.5)
    old = lp - np.log(np.array([[1.5, 0.5, 1.5, 0.5]]))
    adv = np.array([[1.0, 1.0, -1.0, -1.0]])
    loss, _, g, _ = O.policy_loss(x, np.zeros((1, 4), int), old, None, adv)
    assert np.allclose(g, [[0.0, -0.5, 1.5, 0.0]])
    assert np.isclose(loss, -1.2 - 0.5 + 1.5 + 0.8)


# ------------------------------------------------------------ refusals

NULL = None
ANY = ctypes.c_void_p(4096)  # never read: every call below is refused first


def tokens(L, T=2, B=3, I=4, V=5, dtype=0):
    return ctypes.byref(L.Tokens(T, B, I, V, dtype))


@pytest.mark.parametrize("sizes,code", [
    (dict(T=0), -1), (dict(B=0), -1), (dict(I=0), -1), (dict(V=0), -1), (dict(T=-1), -1),
    (dict(dtype=2), -2), (dict(T=65536, B=32768), -2), (dict(V=1 << 30, B=2), -2),
    (dict(V=1 << 30, I=2), -2), (dict(T=1 << 20, B=1 << 10, V=1 << 11), -2)])
def test_sizes_refused(L, sizes, code):
    lib = L.load()
    d = tokens(L, **sizes)
    assert lib.lstmss_loss_workspace_bytes(d) == code
    if "dtype" not in sizes:
        assert lib.lstmss_embed_grad_workspace_bytes(d) == code
    assert lib.lstmss_embed(d, ANY, ANY, 1.0, NULL, ANY, NULL) == code
    assert lib.lstmss_token_logp(d, ANY, ANY, ANY, ANY, 1 << 40, NULL) == code
    assert lib.lstmss_last_error()


def test_most_tokens(L):
    # the token kernel's grid: 256 threads for 16 tokens, below 2^32 of them
    most = (1 << 28) - 16
    lib = L.load()
    assert lib.lstmss_loss_workspace_bytes(tokens(L, T=1, B=most, I=1, V=1)) > 0
    for B in range(most + 1, most + 16):
        assert lib.lstmss_loss_workspace_bytes(tokens(L, T=1, B=B, I=1, V=1)) == -2


def test_null_pointers_refused(L):
    lib, d = L.load(), tokens(L)
    q = ctypes.byref(L.Policy(0.2, 0.2, 0.0, 1.0))
    drop = ctypes.byref(L.drop(0.5, 1))
    big = 1 << 40
    assert lib.lstmss_embed(NULL, ANY, ANY, 1.0, NULL, ANY, NULL) == -1
    for k in range(3):
        a = [ANY] * 3
        a[k] = NULL
        assert lib.lstmss_embed(d, a[0], a[1], 1.0, NULL, a[2], NULL) == -1
        assert lib.lstmss_embed_grad(d, a[0], a[1], 1.0, NULL, 0, a[2], ANY, big, NULL) == -1
        assert lib.lstmss_token_logp(d, a[0], a[1], a[2], ANY, big, NULL) == -1
    for k in range(2):
        a = [ANY] * 2
        a[k] = NULL
        assert lib.lstmss_dropout(8, 0, drop, a[0], a[1], NULL) == -1
        assert lib.lstmss_xent(d, a[0], a[1], NULL, 1.0, ANY, ANY, ANY, ANY, big, NULL) == -1
        assert lib.lstmss_policy_loss(d, q, a[0], a[1], NULL, NULL, ANY, NULL, ANY, ANY, ANY, ANY, big, NULL) == -1
    assert lib.lstmss_dropout(8, 0, NULL, ANY, ANY, NULL) == -1
    assert lib.lstmss_policy_loss(d, NULL, ANY, ANY, NULL, NULL, ANY, NULL, ANY, ANY, ANY, ANY, big, NULL) == -1
    assert lib.lstmss_policy_loss(d, q, ANY, ANY, NULL, NULL, NULL, NULL, ANY, ANY, ANY, ANY, big, NULL) == -1


def test_workspace_refused(L):
    lib, d = L.load(), tokens(L)
    n, m = lib.lstmss_embed_grad_workspace_bytes(d), lib.lstmss_loss_workspace_bytes(d)
    assert n > 0 and m > 0
    for ws, have in ((NULL, n), (ANY, n - 1), (ANY, 0)):
        assert lib.lstmss_embed_grad(d, ANY, ANY, 1.0, NULL, 0, ANY, ws, have, NULL) == -3
    for ws, have in ((NULL, m), (ANY, m - 1)):
        assert lib.lstmss_xent(d, ANY, ANY, NULL, 1.0, ANY, ANY, ANY, ws, have, NULL) == -3
        assert lib.lstmss_token_logp(d, ANY, ANY, ANY, ws, have, NULL) == -3
    assert lib.lstmss_token_logp(d, ANY, ANY, ANY, ctypes.c_void_p(4100), m, NULL) == -1


@pytest.mark.parametrize("drop,code", [((1.0, 1), -1), ((-0.1, 1), -1), ((float("nan"), 1), -1),
                                       ((0.5, 1, 4), -1), ((0.5, 1, 0, -1), -1)])
def test_drop_refused(L, drop, code):
    lib, d = L.load(), tokens(L)
    p = ctypes.byref(L.drop(*drop))
    assert lib.lstmss_dropout(8, 0, p, ANY, ANY, NULL) == code
    assert lib.lstmss_embed(d, ANY, ANY, 1.0, p, ANY, NULL) == code
    assert lib.lstmss_embed_grad(d, ANY, ANY, 1.0, p, 0, ANY, ANY, 1 << 40, NULL) == code


@pytest.mark.parametrize("scale", [float("inf"), -float("inf"), float("nan")])
def test_embedding_scale_refused(L, scale):
    """A column of padding is zero: 0 times such a scale would not be."""
    assert L.load().lstmss_embed(tokens(L), ANY, ANY, scale, NULL, ANY, NULL) == -1


def test_dropout_sizes_refused(L):
    lib, p = L.load(), ctypes.byref(L.drop(0.5, 1))
    assert lib.lstmss_dropout(0, 0, p, ANY, ANY, NULL) == -1
    assert lib.lstmss_dropout(-5, 0, p, ANY, ANY, NULL) == -1
    assert lib.lstmss_dropout(1 << 40, 0, p, ANY, ANY, NULL) == -2
    assert lib.lstmss_dropout(8, 2, p, ANY, ANY, NULL) == -2


@pytest.mark.parametrize("q", [(-0.1, 0.2, 0.0, 1.0), (1.1, 0.2, 0.0, 1.0), (0.2, -0.1, 0.0, 1.0),
                               (0.2, float("inf"), 0.0, 1.0), (0.2, 0.2, -1.0, 1.0),
                               (0.2, 0.2, 0.1, 1.0), (0.2, 0.2, float("nan"), 1.0),
                               (0.2, 0.2, 0.0, float("nan")), (0.2, 0.2, 0.0, float("inf"))])
def test_policy_refused(L, q):
    # the sixth: a KL term without logp_ref
    rc = L.load().lstmss_policy_loss(tokens(L), ctypes.byref(L.Policy(*q)), ANY, ANY, NULL, NULL, ANY,
                                     NULL, ANY, ANY, ANY, ANY, 1 << 40, NULL)
    assert rc == -1


def test_binding_refuses_host_tensors(L):
    import torch
    x = torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError):
        L.embed(x, torch.zeros(4, 5))
    with pytest.raises(ValueError):
        L.dropout(torch.zeros(8), L.drop(0.5, 1))
    with pytest.raises(ValueError):
        L.xent(torch.zeros(2, 5, 3), x)
    with pytest.raises(TypeError):
        L.dropout(None, L.drop(0.5, 1))
    for bad in (dict(offset=-8), dict(offset=2**64), dict(period=2**63)):
        with pytest.raises(ValueError):
            L.drop(0.5, 1, **bad)
    with pytest.raises(ValueError):
        L.loss_workspace_bytes(1, 2**32 + 1, 5)
