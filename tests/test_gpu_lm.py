"""GPU: the language model of the package's operators and layers against the
same model written with elementary torch operations in fp64 on the CPU, whose
gradients automatic differentiation gives; the dropout masks come from the
oracle.  fp32 gradients within the layers' parity bound of 1e-5 (rel. L2), twice
it for those that pass two layers' backward calls and the vocabulary product."""
import numpy as np
import pytest
import torch

from oracle import language as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1806_00512_amd.lm as lm
    return lm


def masks(cfg, drawn):
    out = []
    for l in range(cfg.layers + 1):
        n = cfg.features if l == 0 else cfg.hidden
        size = cfg.steps * n * cfg.batch
        k = O.keep(size, cfg.dropout, cfg.seed, drawn).reshape(cfg.steps, n, cfg.batch)
        out.append(torch.from_numpy(k * O.keep_scale(cfg.dropout)))
        drawn += -(-size // 8) * 8
    return out


def reference(cfg, E, Ws, bs, Wv, tokens, drop):
    """log softmax [T][V][B] in fp64, batch-last as the package has it."""
    x = E[tokens.clamp(min=0)] * cfg.features ** 0.5
    x = (x * (tokens >= 0)[..., None]).permute(0, 2, 1) * drop[0]
    H = cfg.hidden
    for l in range(cfg.layers):
        h = c = torch.zeros(H, cfg.batch, dtype=torch.float64)
        outs = []
        for t in range(cfg.steps):
            a = Ws[l] @ torch.cat([x[t], h]) + bs[l][:, None]
            i, f, g, o = a[:H].sigmoid(), a[H:2 * H].sigmoid(), a[2 * H:3 * H].tanh(), a[3 * H:].sigmoid()
            c = f * c + i * g
            h = o * c.tanh()
            outs.append(h)
        x = torch.stack(outs) * drop[l + 1]
    return torch.log_softmax(torch.stack([Wv @ x[t] for t in range(cfg.steps)]), 1)


def rel(a, b):
    return float((a.double().cpu() - b).norm() / b.norm())


def picked(lsm, targets):
    return torch.where(targets >= 0, lsm.gather(1, targets.clamp(min=0)[:, None])[:, 0], 0.0)


@pytest.mark.parametrize("T,B,I,H,V,layers", [(5, 8, 24, 32, 40, 2), (7, 20, 36, 40, 130, 1), (1, 3, 8, 16, 5, 2)])
def test_gradients(M, T, B, I, H, V, layers):
    cfg = M.LanguageConfig(vocabulary=V, features=I, hidden=H, layers=layers, batch=B, steps=T, dropout=0.3, seed=5)
    E, Ws, bs, Wv = M.make_weights(cfg)
    bs = [b + 0.1 * torch.randn(b.shape, device=DEV) for b in bs]
    model = M.LanguageModel(cfg, E, Ws, bs, Wv)
    tokens, targets = M.synthetic_batch(cfg, 3)
    leaves = [t.double().cpu().requires_grad_() for t in [E, *Ws, *bs, Wv]]
    drop = masks(cfg, model.drawn)
    lsm = reference(cfg, leaves[0], leaves[1:1 + layers], leaves[1 + layers:1 + 2 * layers], leaves[-1],
                    tokens.cpu().long(), drop)
    loss = -picked(lsm, targets.cpu().long()).sum() / (T * B)
    loss.backward()
    got = model.step(tokens, targets, update=False)
    assert abs(float(got) - float(loss.detach())) < 1e-5 * abs(float(loss.detach()))
    grads = [model.dE, *[o["dW"] for o in model.outs], *[o["db"] for o in model.outs], model.dWv]
    for g, leaf in zip(grads, leaves):
        assert rel(g, leaf.grad) < 2e-5
    # the update, and the next step's masks are others
    before = [t.clone() for t in [model.E, model.Wv, *model.Ws]]
    model.update()
    for b, t, g in zip(before, [model.E, model.Wv, *model.Ws], [model.dE, model.dWv, *[o["dW"] for o in model.outs]]):
        assert rel(t, b.double().cpu() - cfg.lr * g.double().cpu()) < 1e-6
    assert not torch.equal(masks(cfg, model.drawn)[0], drop[0])


def test_policy_gradients(M):
    T, B, V = 6, 10, 50
    cfg = M.LanguageConfig(vocabulary=V, features=16, hidden=24, layers=2, batch=B, steps=T, dropout=0.3, seed=6)
    model = M.LanguageModel(cfg, *M.make_weights(cfg))
    tokens, targets = M.synthetic_batch(cfg, 4)
    leaves = [t.double().cpu().requires_grad_() for t in [model.E, *model.Ws, *model.bs, model.Wv]]
    ones = [torch.ones(1, dtype=torch.float64)] * 3
    lsm = reference(cfg, leaves[0], leaves[1:3], leaves[3:5], leaves[5], tokens.cpu().long(), ones)
    y = targets.cpu().long()
    lp = picked(lsm, y)
    score = model.score(tokens, targets)
    assert (score.double().cpu() - lp).abs().max() < 1e-5
    g = torch.Generator().manual_seed(1)
    r = torch.rand((T, B), generator=g, dtype=torch.float64) - 0.5
    r = torch.where(((r - np.log(0.8)).abs() < 1e-2) | ((r - np.log(1.2)).abs() < 1e-2), 0.0, r)
    old, ref = (lp.detach() - r).float(), (lp.detach() + 0.1).float()
    adv = torch.randn((T, B), generator=g)
    ratio = torch.exp(lp - old.double())
    q = ref.double() - lp
    each = -torch.minimum(ratio * adv, ratio.clamp(0.8, 1.2) * adv) + 0.05 * (torch.exp(q) - q - 1)
    loss = torch.where(y >= 0, each, 0.0).sum() / (T * B)
    loss.backward()
    got = model.policy_step(tokens, targets, old.to(DEV), ref.to(DEV), adv.to(DEV), kl=0.05, update=False)
    assert abs(float(got) - float(loss.detach())) < 1e-5
    grads = [model.dE, *[o["dW"] for o in model.outs], *[o["db"] for o in model.outs], model.dWv]
    for g, leaf in zip(grads, leaves):
        assert rel(g, leaf.grad) < 2e-5


def test_example_trains(M):
    losses, moved = M.main(60)
    assert losses[0] > 0.7 * np.log(200) and losses[-1] < 0.8 * losses[0]
    assert float(moved[::2].mean()) > float(moved[1::2].mean())


def test_bf16_step(M):
    cfg = M.LanguageConfig(vocabulary=120, features=32, hidden=48, layers=2, batch=16, steps=6, dropout=0.2,
                           dtype=torch.bfloat16)
    E, Ws, bs, Wv = M.make_weights(cfg)
    model = M.LanguageModel(cfg, E, Ws, bs, Wv)
    tokens, targets = M.synthetic_batch(cfg, 7)
    leaves = [t.double().cpu().requires_grad_() for t in [E, *Ws, *bs, Wv]]
    lsm = reference(cfg, leaves[0], leaves[1:3], leaves[3:5], leaves[5], tokens.cpu().long(), masks(cfg, 0))
    loss = -picked(lsm, targets.cpu().long()).sum() / (6 * 16)
    loss.backward()
    got = model.step(tokens, targets, sparse=False, update=False)
    assert abs(float(got) - float(loss.detach())) < 2e-2 * float(loss.detach())
    for g, leaf in zip([model.dE, model.outs[0]["dW"], model.outs[1]["dW"], model.dWv],
                       [leaves[0], leaves[1], leaves[2], leaves[5]]):
        assert rel(g, leaf.grad) < 4e-2     # the layers' bf16 bound, twice
    assert torch.isfinite(model.step(tokens, targets, sparse=True))


def test_bf16_vocabulary_products_are_summed_in_fp32(M):
    """The vocabulary's gradient and the top layer's, from the gradient in the logits and the
    activations as they are stored.  A product of two bf16 numbers is exact in fp32, so only the
    additions round: within 2^-23 of the terms' sizes each, in any order, by either rounding."""
    T, B, V = 5, 4, 40
    cfg = M.LanguageConfig(vocabulary=V, features=16, hidden=24, layers=1, batch=B, steps=T, dropout=0.0,
                           dtype=torch.bfloat16)
    model = M.LanguageModel(cfg, *M.make_weights(cfg))
    model.step(*M.synthetic_batch(cfg, 8), update=False)
    d, top, Wv = (t.double().cpu() for t in (model.logits, model.top, model.Wv))
    want = sum(d[t] @ top[t].t() for t in range(T))
    size = sum(d[t].abs() @ top[t].t().abs() for t in range(T))
    assert ((model.dWv.double().cpu() - want).abs() <= (B + T) * 2.0**-23 * size + 2.0**-126).all()
    for t in range(T):
        size = Wv.t().abs() @ d[t].abs()
        assert ((model.dH[t].double().cpu() - Wv.t() @ d[t]).abs() <= V * 2.0**-23 * size + 2.0**-126).all()


def test_shapes_refused(M):
    cfg = M.LanguageConfig(vocabulary=20, features=8, hidden=16, layers=1, batch=2, steps=2)
    E, Ws, bs, Wv = M.make_weights(cfg)
    for bad in ((E[:-1], Ws, bs, Wv), (E, Ws, bs, Wv[:, :-1]), (E, [Ws[0][:-1]], bs, Wv), (E.double(), Ws, bs, Wv)):
        with pytest.raises(ValueError):
            M.LanguageModel(cfg, *bad)
