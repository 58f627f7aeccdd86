"""GPU: beam search against its definition in 64 bits.  Tokens, parents and finished beams are
equal, wherever two candidates' scores in 64 bits are further apart than the kernel's own
rounding: 2^-21 (its softmax's sum is of fp32 exponentials, each within 8 * 2^-24; the same beam's
candidates are shifted alike).  Inputs are drawn without such pairs.  Scores: that, and one
rounding to fp32."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NEAR = 2.0**-21


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1806_00512_amd.lstmss as lstmss
    lstmss.load()
    return lstmss


def reference(logits, scores, K, eos=-1, done=None):
    """(scores, tokens, parents, done) [N] by definition, and the smallest distance between two
    neighbours of different beams among the K + 1 first of a sequence."""
    x = logits.detach().float().cpu().numpy().astype(np.float64)
    V, N = x.shape
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, np.finfo(np.float32).max))
    sc = scores.cpu().numpy().astype(np.float64)
    sc = np.where(np.isnan(sc), -np.inf, sc)
    dn = np.zeros(N, int) if done is None else done.cpu().numpy()
    cand = np.full((V, N), -np.inf)
    for n in range(N):
        if dn[n]:
            cand[eos, n] = sc[n]
            continue
        m = x[:, n].max()
        if m > -np.inf and sc[n] > -np.inf:
            cand[:, n] = sc[n] - np.log(np.exp(x[:, n] - m).sum()) + (x[:, n] - m)
    out = [np.full(N, -np.inf), np.full(N, -1), np.zeros(N, int), np.zeros(N, int)]
    gap = np.inf
    for s in range(N // K):
        flat = cand[:, s * K:(s + 1) * K].T.reshape(-1)
        order = np.argsort(-flat, kind="stable")[:K + 1]
        for a, b in zip(order[:-1], order[1:]):
            if flat[b] > -np.inf and a // V != b // V:
                gap = min(gap, flat[a] - flat[b])
        for j in range(K):
            n = s * K + j
            if j < len(order) and flat[order[j]] > -np.inf:
                k, v = divmod(int(order[j]), V)
                out[0][n], out[1][n], out[2][n] = flat[order[j]], v, k
                out[3][n] = int(dn[s * K + k] != 0 or v == eos)
            else:
                out[2][n] = j
    return out, gap


def check(L, logits, scores, K, eos=-1, done=None):
    ref, gap = reference(logits, scores, K, eos, done)
    assert gap > NEAR, "the inputs have a pair that a rounding decides"
    o = L.beam_step(logits, scores, K, eos=eos, done=done)
    assert set(o) == {"scores", "tokens", "parents"} | ({"done"} if eos >= 0 else set())
    assert np.array_equal(o["tokens"].cpu().numpy(), ref[1])
    assert np.array_equal(o["parents"].cpu().numpy(), ref[2])
    if eos >= 0:
        assert np.array_equal(o["done"].cpu().numpy(), ref[3])
    got = o["scores"].cpu().numpy().astype(np.float64)
    there = ref[0] > -np.inf
    assert np.array_equal(got > -np.inf, there)
    got, want = got[there], ref[0][there]
    assert (np.abs(got - want) <= NEAR + 2.0**-24 * np.abs(want)).all()
    return o


SIZES = [  # S, K, V
    (1, 1, 1), (1, 1, 700), (1, 4, 10000), (2, 3, 5), (5, 5, 63), (3, 7, 64), (3, 4, 65), (13, 5, 5003), (64, 8, 1000),
    (1, 32, 300), (2, 32, 3), (40, 2, 129), (9, 16, 2000), (300, 1, 130), (1, 6, 200001), (2, 2, 70000), (33, 3, 257)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S,K,V", SIZES)
@pytest.mark.parametrize("kind", ["plain", "ends"])
def test_step(L, dtype, S, K, V, kind):
    g = torch.Generator(device=DEV)
    N, eos, done = S * K, -1, None
    for seed in range(100):  # inputs without near pairs
        g.manual_seed(1000 * K + V + 7 * seed)
        logits = (torch.randn(V, N, generator=g, device=DEV) * 3).to(TYPES[dtype])
        scores = -torch.rand(N, generator=g, device=DEV) * 9
        if kind == "ends":
            eos = V // 2
            done = (torch.rand(N, generator=g, device=DEV) < 0.3).int() * 5
            logits[torch.rand(V, N, generator=g, device=DEV) < 0.3] = -math.inf
        if reference(logits, scores, K, eos, done)[1] > NEAR:
            break
    check(L, logits, scores, K, eos, done)
    # the first step: one beam of each sequence
    first = torch.where(torch.arange(N, device=DEV) % K == K // 2, 0.0, -math.inf)
    check(L, logits, first, K, eos, None if done is None else torch.zeros_like(done))


def test_ties_go_to_the_lowest(L):
    """Equal logits within a beam, and equal beams: whole columns the same."""
    for S, K, V in ((2, 4, 300), (1, 8, 5000), (3, 3, 64)):
        col = torch.randn(V, 1, device=DEV).bfloat16().float().round()
        logits = col.expand(V, S * K).contiguous()
        o = L.beam_step(logits, torch.full((S * K,), -1.0, device=DEV), K)
        # by (score, k, v): the largest logit's tokens of beam 0, then those of beam 1, ...
        c = col[:, 0].cpu().numpy()
        order = sorted(((-c[v], k, v) for k in range(K) for v in range(V)))[:K]
        assert o["tokens"].tolist() == [v for _, _, v in order] * S
        assert o["parents"].tolist() == [k for _, k, _ in order] * S
    same = torch.zeros(1000, 4, device=DEV)
    o = L.beam_step(same, torch.zeros(4, device=DEV), 4)
    assert o["tokens"].tolist() == [0, 1, 2, 3] and o["parents"].tolist() == [0] * 4
    # scores so far from zero that they are all one number
    o = L.beam_step(torch.randn(1000, 4, device=DEV), torch.full((4,), -1e30, device=DEV), 4)
    assert o["tokens"].tolist() == [0, 1, 2, 3] and o["parents"].tolist() == [0] * 4


@pytest.mark.parametrize("S,K,V", [(1, 4, 40000), (3, 8, 20000), (1, 32, 100000), (2, 1, 70000)])
@pytest.mark.parametrize("size", [1e-25, 1.0])
def test_scores_that_64_bits_do_not_tell_apart(L, S, K, V, size):
    """Different logits, equal scores: the lowest tokens of the lowest beam, many groups of them."""
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    logits = size * torch.randn(V, S * K, generator=g, device=DEV)
    scores = torch.full((S * K,), -1e30, device=DEV) if size == 1.0 else -2.0 * torch.arange(
        K, device=DEV, dtype=torch.float32).repeat(S)
    o = L.beam_step(logits, scores, K)
    assert o["tokens"].tolist() == list(range(K)) * S and o["parents"].tolist() == [0] * (K * S)


def test_negative_zero_is_a_tie(L):
    """A finished beam of score -0 before one of score 0 that has one token alone."""
    logits = torch.full((100, 4), -math.inf, device=DEV)
    logits[7, 1:] = 0.0
    scores = torch.tensor([-0.0, 0.0, -1.0, -2.0], device=DEV)
    done = torch.tensor([1, 0, 0, 0], dtype=torch.int32, device=DEV)
    o = L.beam_step(logits, scores, 4, eos=3, done=done)
    assert o["parents"].tolist() == [0, 1, 2, 3] and o["tokens"].tolist() == [3, 7, 7, 7]
    assert o["scores"].tolist() == [0.0, 0.0, -1.0, -2.0] and o["done"].tolist() == [1, 0, 0, 0]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_and_odd_values(L, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    S, K, V = 6, 4, 333
    N = S * K
    logits = torch.randn(V, N, generator=g, device=DEV).to(TYPES[dtype])
    scores = -torch.rand(N, generator=g, device=DEV) * 3
    logits[:, 0] = -math.inf                       # a beam without tokens
    logits[:, 4:8] = -math.inf                     # a sequence without tokens
    logits[7:, 8:12] = -math.inf                   # few of them
    logits[2:, 12:16] = -math.inf
    logits[5, 16] = math.nan                       # as if it were not there
    logits[::3, 17] = math.nan
    logits[9, 18] = math.inf                       # takes all
    logits[10, 19] = torch.finfo(logits.dtype).min
    logits[:, 20] = torch.finfo(logits.dtype).min  # masks that are finite: evenly spread
    scores[3], scores[21] = math.nan, -math.inf
    check(L, logits, scores, K)
    done = torch.zeros(N, dtype=torch.int32, device=DEV)
    done[0], done[5], done[12:16], done[21], done[23] = 1, 1, 1, 1, 1
    check(L, logits, scores, K, eos=332, done=done)
    one = torch.full((1, N), 3.0, device=DEV, dtype=logits.dtype)
    check(L, one, scores, K, eos=0)


def test_more_equal_candidates_than_the_list_holds(L):
    """One group of tokens of one beam: 2048 of them, every 32nd thread's far below the others, so
    that the bound by which the kernel lists candidates keeps nearly all of them."""
    V, K = 524288, 32
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    logits = torch.full((V, K), -math.inf, device=DEV)
    at = torch.arange(4096, 4096 + 2048, device=DEV)
    x = torch.randn(2048, generator=g, device=DEV)
    x[(torch.arange(2048, device=DEV) % 1024) >= 992] -= 50.0
    logits[at, 3] = x
    scores = torch.full((K,), -math.inf, device=DEV)
    scores[3] = -1.0
    o = L.beam_step(logits, scores, K)
    order = torch.sort(x, descending=True, stable=True).indices[:K]
    assert torch.equal(o["tokens"], (at[order]).int()) and (o["parents"] == 3).all()
    lp = torch.log_softmax(x.double(), 0)[order] - 1.0
    assert float((o["scores"].double() - lp).abs().max()) < 2e-6
    # the same for groups: one beam's
    logits[:, 3] = torch.randn(V, generator=g, device=DEV)
    o = L.beam_step(logits, scores, K)
    order = torch.sort(logits[:, 3], descending=True, stable=True).indices[:K]
    assert torch.equal(o["tokens"], order.int())


def test_offsets_past_31_bits(L):
    S, K, V = 4096, 8, 70000
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    logits = torch.empty((V, S * K), dtype=torch.bfloat16, device=DEV)
    assert logits.numel() > 2**31
    for v in range(0, V, 10000):
        logits[v:v + 10000] = torch.randn(10000, S * K, generator=g, device=DEV) * 3
    scores = -torch.rand(S * K, generator=g, device=DEV) * 5
    o = L.beam_step(logits, scores, K)
    compared = 0
    for s in (0, 1, 2047, S - 3, S - 2, S - 1):
        cols = slice(s * K, (s + 1) * K)
        ref, gap = reference(logits[:, cols], scores[cols], K)
        if gap > NEAR:
            compared += 1
            assert np.array_equal(o["tokens"][cols].cpu().numpy(), ref[1])
            assert np.array_equal(o["parents"][cols].cpu().numpy(), ref[2])
    assert compared >= 4


def test_in_place_and_replayed(L):
    S, K, V = 5, 4, 3000
    N = S * K
    logits, scores = torch.randn(V, N, device=DEV), -torch.rand(N, device=DEV)
    done = torch.zeros(N, dtype=torch.int32, device=DEV)
    want = L.beam_step(logits, scores, K, eos=2, done=done)
    s, d = scores.clone(), done.clone()
    o = L.beam_step(logits, s, K, eos=2, done=d, out={"scores": s, "done": d})
    assert o["scores"] is s and all(torch.equal(o[k], want[k]) for k in want)
    ws = torch.empty(L.beam_workspace_bytes(S, K, V), dtype=torch.uint8, device=DEV)
    states, moved = torch.randn(3, 50, N, device=DEV), torch.empty(3, 50, N, device=DEV)

    def calls():
        L.beam_step(logits, scores, K, eos=2, done=done, out=o, ws=ws)
        L.beam_reorder(states, o["parents"], K, out=moved)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        logits.copy_(torch.randn(V, N, device=DEV))
        states.copy_(torch.randn(3, 50, N, device=DEV))
        want = L.beam_step(logits, scores, K, eos=2, done=done)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o[k], want[k]) for k in want)
        assert torch.equal(moved, L.beam_reorder(states, want["parents"], K))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,K", [((1, 1), 1), ((3, 8), 4), ((2, 65, 15), 5), ((4, 1023, 512), 8), ((7, 300), 3),
                                     ((20,), 4), ((5000, 36), 6), ((3, 7, 1000), 1), ((2, 70000, 32), 32)])
def test_reorder(L, dtype, shape, K):
    N = shape[-1]
    x = torch.randn(shape, device=DEV).to(TYPES[dtype])
    p = torch.randint(0, K, (N,), device=DEV, dtype=torch.int32)
    col = torch.arange(N, device=DEV) // K * K + p
    assert torch.equal(L.beam_reorder(x, p, K), x[..., col])
    bad = p.clone()
    bad[::3] = torch.tensor([-1, K, 2**31 - 1, -2**31], dtype=torch.int32, device=DEV).repeat(N)[:bad[::3].numel()]
    out = L.beam_reorder(x, bad, K)
    there = (bad >= 0) & (bad < K)
    assert torch.equal(out, torch.where(there, x[..., col], torch.zeros((), dtype=x.dtype, device=DEV)))


def test_trace(L):
    rng = np.random.default_rng(3)
    for T, S, K in ((1, 1, 1), (7, 3, 4), (30, 50, 8), (4, 1, 32)):
        N = S * K
        tok, par = rng.integers(0, 99, (T, N)).astype(np.int32), rng.integers(0, K, (T, N)).astype(np.int32)
        par[rng.random((T, N)) < 0.02] = rng.choice([-1, K, 2**31 - 1])
        want = np.full((T, N), -1, np.int32)
        for n in range(N):
            at = n
            for t in range(T - 1, -1, -1):
                want[t, n] = tok[t, at]
                if not 0 <= par[t, at] < K:
                    break
                at = n // K * K + par[t, at]
        got = L.beam_trace(torch.from_numpy(tok).to(DEV), torch.from_numpy(par).to(DEV), K)
        assert np.array_equal(got.cpu().numpy(), want)


def test_search_of_several_steps_finds_what_a_search_by_hand_finds(L):
    """Step, reorder and trace over a random chain: token v follows u with logits table[v][u]."""
    g = torch.Generator(device=DEV)
    g.manual_seed(17)
    S, K, V, T, eos = 4, 3, 40, 8, 0
    N = S * K
    table = torch.randn(V, V, generator=g, device=DEV) * 2
    start = torch.randint(1, V, (S,), generator=g, device=DEV)
    tokens = start.repeat_interleave(K).int()
    scores = torch.where(torch.arange(N, device=DEV) % K == 0, 0.0, -math.inf)
    done = torch.zeros(N, dtype=torch.int32, device=DEV)
    state = torch.zeros(5, N, device=DEV)
    toks, pars = [], []
    for _ in range(T):
        logits = table[:, tokens.clamp(min=0).long()].contiguous()
        o = L.beam_step(logits, scores, K, eos=eos, done=done)
        scores, done, tokens = o["scores"], o["done"], o["tokens"]
        state = L.beam_reorder(state, o["parents"], K)
        state[0] += tokens  # what a model would carry along
        toks.append(tokens)
        pars.append(o["parents"])
    paths = L.beam_trace(torch.stack(toks), torch.stack(pars), K).cpu().numpy()
    logp = torch.log_softmax(table.double(), 0).cpu().numpy()
    for s in range(S):
        beams = [(0.0, [int(start[s])], False)]
        for _ in range(T):
            nxt = []
            for sc, p, fin in beams:
                nxt += [(sc, p + [eos], True)] if fin else [(sc + logp[v, p[-1]], p + [v], v == eos) for v in range(V)]
            beams = sorted(nxt, key=lambda b: -b[0])[:K]
        for k, (sc, p, fin) in enumerate(beams):
            n = s * K + k
            assert paths[:, n].tolist() == p[1:]
            assert abs(float(scores[n]) - sc) < 1e-5 * (1 + abs(sc)) and bool(done[n]) == fin
            assert float(state[0, n]) == sum(p[1:])


def test_refusals(L):
    x, s = torch.randn(50, 12, device=DEV), torch.zeros(12, device=DEV)
    d = torch.zeros(12, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        L.beam_step(x, s, 5)
    with pytest.raises(ValueError):
        L.beam_step(x, s, 0)
    with pytest.raises(ValueError):
        L.beam_step(x.t(), s, 4)
    with pytest.raises(ValueError):
        L.beam_step(x, s.double(), 4)
    with pytest.raises(ValueError):
        L.beam_step(x, s, 4, eos=1, done=d.long())
    with pytest.raises(L.LstmssError):
        L.beam_step(x, s, 4, eos=50)
    with pytest.raises(L.LstmssError):
        L.beam_step(x, s, 4, eos=-2)
    with pytest.raises(L.LstmssError):
        L.beam_step(x, s, 4, done=d)
    with pytest.raises(L.LstmssError):
        L.beam_step(torch.randn(5, 66, device=DEV), torch.zeros(66, device=DEV), 33)
    with pytest.raises(L.LstmssError):
        L.beam_step(x, s, 4, ws=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(L.LstmssError):
        L.beam_reorder(x, d, 4, out=x)
    with pytest.raises(ValueError):
        L.beam_reorder(x, d[:6], 4)
    with pytest.raises(ValueError):
        L.beam_trace(d.view(1, 12), d.view(2, 6), 4)
    with pytest.raises(L.LstmssError):
        L.beam_reorder(x[:0], d, 4)


def test_steps_on_two_streams_at_once(L):
    g = torch.Generator(device=DEV)
    g.manual_seed(31)
    ins = []
    for S, K, V in ((5, 4, 9001), (64, 8, 5000)):
        logits = torch.randn(V, S * K, generator=g, device=DEV)
        scores = -torch.rand(S * K, generator=g, device=DEV) * 9
        ins.append((logits, scores, K, L.beam_step(logits, scores, K), torch.cuda.Stream(DEV)))
    torch.cuda.synchronize()
    got = [L.beam_step(x, sc, K, stream=s) for x, sc, K, _, s in ins]
    torch.cuda.synchronize()
    for o, (_, _, _, want, _) in zip(got, ins):
        assert all(torch.equal(o[k], want[k]) for k in want)


@pytest.mark.parametrize("dtype,V", [("f32", 1 << 18), ("f32", 1 << 20), ("bf16", 1 << 22)])
def test_sums_of_many_tokens_keep_their_order(L, dtype, V):
    """32 beams over many tokens, so that a group has 2^10 to 2^14 of them: one token 3, of the
    others of a column 64 in 1024 0 and the rest the same (terms whose rounded sums err in one
    direction), or all slowly rising.  The beams' best candidates are 1e-5 apart and come out in
    their order.

    In units of u = 2^-24 a term's exponential is within 2 (the instruction) + 2.3 d (the
    difference, the constant and their product), d the distances to the references on its way;
    eight terms' sum adds 7, the lane's factor 2 and two roundings, the lanes' sum 6, the group's
    factor 2 and a rounding: 21 u + 2.3 u times the softmax's mean of d.  A reference is the
    largest logit or below it by no more than the rise, which d counts twice then."""
    K, u = 32, 2.0**-24
    g = torch.Generator(device=DEV)
    g.manual_seed(23)
    logits = torch.empty(V, K, dtype=TYPES[dtype], device=DEV)
    v = torch.arange(V, device=DEV, dtype=torch.float64)
    for k in range(K):
        logits[:, k] = v / V - 1.0 if k % 4 == 3 else torch.where(v % 1024 < 64, 0.0, (-1.1, -9.0, -5.3)[k % 4])
        logits[int(torch.randint(0, V, (1,), generator=g, device=DEV)), k] = 3.0
    lse, bound = np.empty(K), np.empty(K)
    for k in range(K):
        x = logits[:, k].double().cpu().numpy()
        e = np.exp(x - 3.0)
        lse[k] = 3.0 + np.log(e.sum())
        bound[k] = u * (21 + 2.3 * ((e * (3.0 - x)).sum() / e.sum() + (2.0 if k % 4 == 3 else 0.0)))
    place = np.array([7 * k % K for k in range(K)])
    scores = torch.from_numpy(lse - 3.0 - 1e-5 * place).float().to(DEV)
    want = scores.cpu().numpy().astype(np.float64) + (3.0 - lse)
    order = np.argsort(-want)
    gaps = want[order][:-1] - want[order][1:]
    assert (gaps > bound[order][:-1] + bound[order][1:]).all()
    o = L.beam_step(logits, scores, K)
    assert o["parents"].tolist() == order.tolist()
    assert o["tokens"].tolist() == logits.argmax(0)[torch.from_numpy(order).to(DEV)].tolist()
    err = np.abs(o["scores"].cpu().numpy().astype(np.float64) - want[order])
    assert (err <= bound[order] + u * np.abs(want[order])).all(), (err / u).max()
