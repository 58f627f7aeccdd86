"""A recurrent language model on the package's kernels: token ids in, loss and
updated weights out.

  embedding lookup (scaled, with dropout), a stack of LSTM layers with dropout
  between them and on top, a product with the vocabulary's rows, cross entropy
  (or the clipped policy loss), and all of it backward, the LSTM layers with
  the structurally sparsified backward pass in the sparse steps of a
  dense-after-sparse schedule (section 5).

Every dropout of a step has its own stretch of the counter-based generator, so
the backward pass asks for the same mask again and none is stored.

With a bias on the vocabulary (head_bias) or a residual block of two linear
layers between the stack and it (block > 0: top + W2 gelu(W1 top + b1) + b2) the
head is of linear and linear_grad calls.  Without either the vocabulary product
is a plain matrix product of one step at a time (torch), and models that were
trained so go on bit for bit.  Weights are updated by SGD or, those of the layers
and of the block with optimizer "muon", by orthogonalised momentum; generate()
answers prompts by beam search.

The rest are liblstmss calls, a training step's on buffers allocated once (generate()
allocates what an answer takes, step by step).  `python -m
paper_1806_00512_amd.lm` trains a small model on synthetic sequences and lets it
answer.
"""
from __future__ import annotations

import math
from dataclasses import dataclass

import torch

from . import lstmss as L


@dataclass
class LanguageConfig:
    vocabulary: int
    features: int                  # of the embedding
    hidden: int
    layers: int
    batch: int
    steps: int
    dtype: torch.dtype = torch.float32
    lr: float = 0.5
    dropout: float = 0.5
    seed: int = 1
    sparsity: float = 0.5
    P: int = 4
    R: int = 8
    head_bias: bool = False
    block: int = 0                 # features between the two layers of the residual block
    optimizer: str = "sgd"         # or "muon"
    muon_lr: float = 0.02
    momentum: float = 0.95

    def layer_input(self, l: int) -> int:
        return self.features if l == 0 else self.hidden

    def head_shapes(self) -> dict:
        """Shapes of what the head has besides Wv; biases (one number) are fp32."""
        out = {}
        if self.block > 0:
            out.update(W1=(self.block, self.hidden), b1=(self.block,), W2=(self.hidden, self.block),
                       b2=(self.hidden,))
        if self.head_bias:
            out["bv"] = (self.vocabulary,)
        return out


def _product(a, b):
    """a @ b in fp32, whatever the storage type: a gradient's terms are not rounded to bf16
    before they are summed."""
    return torch.mm(a, b) if a.dtype == torch.float32 else torch.mm(a, b, out_dtype=torch.float32)


class LanguageModel:
    """Weights E [V][I], Ws[l] [4H][I_l + H], bs[l] [4H] (fp32), Wv [V][H] and `head`, a dict of
    what cfg.head_shapes() names; all but the biases in the storage type.  step() and
    policy_step() train them in place."""

    def __init__(self, cfg: LanguageConfig, E, Ws, bs, Wv, device="cuda:0", head=None):
        L.load()
        self.cfg, self.E, self.Ws, self.bs, self.Wv = cfg, E, list(Ws), list(bs), Wv
        self.head = dict(head or {})
        if {k: tuple(v.shape) for k, v in self.head.items()} != cfg.head_shapes():
            raise ValueError("head must be of %s" % (cfg.head_shapes(),))
        if cfg.optimizer not in ("sgd", "muon"):
            raise ValueError("optimizer %r is neither sgd nor muon" % (cfg.optimizer,))
        dev, dt, f32 = torch.device(device), cfg.dtype, torch.float32
        T, B, H, V, I = cfg.steps, cfg.batch, cfg.hidden, cfg.vocabulary, cfg.features
        if tuple(E.shape) != (V, I) or tuple(Wv.shape) != (V, H) or E.dtype != dt or Wv.dtype != dt:
            raise ValueError("E must be [%d][%d] and Wv [%d][%d], both %s" % (V, I, V, H, dt))
        self.scale = math.sqrt(I)
        self.drawn = 0             # mask elements that earlier steps took
        e = dict(device=dev)
        self.inputs, self.houts, self.caches, self.fws, self.outs = [], [], [], [], []
        ws = 0
        for l in range(cfg.layers):
            n = cfg.layer_input(l)
            if tuple(self.Ws[l].shape) != (4 * H, n + H) or self.Ws[l].dtype != dt:
                raise ValueError("W[%d] must be [%d][%d] %s" % (l, 4 * H, n + H, dt))
            d = L.dims(T, B, n, H, dt)
            self.inputs.append(torch.empty((T, n, B), dtype=dt, **e))
            self.houts.append(torch.empty((T, H, B), dtype=dt, **e))
            self.caches.append(torch.empty(L.cache_bytes(d), dtype=torch.uint8, **e))
            self.fws.append(torch.empty(L.fwd_workspace_bytes(d), dtype=torch.uint8, **e))
            self.outs.append({"dX": torch.empty((T, n, B), dtype=f32, **e)})
            s = L.structure(cfg.P, cfg.R)
            ws = max(ws, L.workspace_bytes(d, 0.0), L.workspace_bytes(d, cfg.sparsity, s))
        self.ws = torch.empty(ws, dtype=torch.uint8, **e)
        self.top = torch.empty((T, H, B), dtype=dt, **e)
        self.logits = torch.empty((T, V, B), dtype=dt, **e)
        self.loss_out = {"loss": torch.empty(1, dtype=f32, **e), "logp": torch.empty((T, B), dtype=f32, **e),
                         "dlogits": self.logits}
        self.loss_ws = torch.empty(L.loss_workspace_bytes(T, B, V, dt), dtype=torch.uint8, **e)
        self.dH = torch.empty((T, H, B), dtype=f32, **e)
        self.dWv = torch.empty((V, H), dtype=f32, **e)
        self.dE = torch.empty((V, I), dtype=f32, **e)
        self.dE_ws = torch.empty(L.embed_grad_workspace_bytes(T, B, I, V), dtype=torch.uint8, **e)
        if self.head:
            self._head_buffers(e)
        self.moments = {}
        if cfg.optimizer == "muon":
            rows = [(W.shape[0], W.shape[1], 4) for W in self.Ws] + \
                [(*self.head[k].shape, 1) for k in ("W1", "W2") if k in self.head]
            self.muon_ws = torch.empty(max(L.muon_workspace_bytes(*r) for r in rows), dtype=torch.uint8, **e)

    def _head_buffers(self, e):
        """What the head's linear layers write: in self.act the block's inner pre-activations z,
        activations a and outputs y, in self.grads the gradients."""
        cfg = self.cfg
        T, B, H, V, F, dt = cfg.steps, cfg.batch, cfg.hidden, cfg.vocabulary, cfg.block, cfg.dtype
        sizes = [L.linear_workspace_bytes(T, B, H, V, dt), L.linear_grad_workspace_bytes(T, B, H, V, dt)]
        self.act = {}
        if F > 0:
            self.act = {k: torch.empty((T, n, B), dtype=dt, **e) for k, n in (("z", F), ("a", F), ("y", H))}
            self.da, self.dtop = torch.empty((T, F, B), **e), torch.empty((T, H, B), **e)
            sizes += [L.linear_workspace_bytes(T, B, H, F, dt), L.linear_workspace_bytes(T, B, F, H, dt),
                      L.linear_grad_workspace_bytes(T, B, H, F, dt, act="gelu", dY_dtype=L.F32),
                      L.linear_grad_workspace_bytes(T, B, F, H, dt, dY_dtype=L.F32)]
        self.grads = {k: torch.empty(shape, **e) for k, shape in cfg.head_shapes().items()}
        self.head_ws = torch.empty(max(sizes), dtype=torch.uint8, **e)

    def _head(self, top, logits=None, keep=None, ws=None):
        """Logits of the stack's outputs top [T][H][B] by linear calls; keep: z, a and y to write."""
        h, keep = self.head, keep or {}
        if self.cfg.block > 0:
            a = L.linear(top, h["W1"], h["b1"], act="gelu", z=keep.get("z"), out=keep.get("a"), ws=ws)
            top = L.linear(a, h["W2"], h["b2"], res=top, out=keep.get("y"), ws=ws)
        return L.linear(top, self.Wv, h.get("bv"), out=logits, ws=ws)

    def _head_backward(self):
        """dH, dWv and the head's own gradients from dL/dlogits in the logits' place."""
        cfg, g, h, ws = self.cfg, self.grads, self.head, self.head_ws
        block = cfg.block > 0
        want = ("dX", "dW", "db") if cfg.head_bias else ("dX", "dW")
        L.linear_grad(self.act["y"] if block else self.top, self.Wv, self.logits, want=want,
                      out={"dX": self.dH, "dW": self.dWv, "db": g.get("bv")}, ws=ws)
        if block:
            L.linear_grad(self.act["a"], h["W2"], self.dH, out={"dX": self.da, "dW": g["W2"], "db": g["b2"]}, ws=ws)
            L.linear_grad(self.top, h["W1"], self.da, act="gelu", z=self.act["z"],
                          out={"dX": self.dtop, "dW": g["W1"], "db": g["b1"]}, ws=ws)
            self.dH += self.dtop

    def _drops(self, training: bool):
        """A dropout for the embedding and one for every layer's output, or Nones; the
        step's share of the generator is taken whether it is used or not."""
        cfg, out = self.cfg, []
        for l in range(cfg.layers + 1):
            n = cfg.steps * cfg.batch * (cfg.features if l == 0 else cfg.hidden)
            out.append(L.drop(cfg.dropout, cfg.seed, self.drawn) if training and cfg.dropout > 0 else None)
            self.drawn += -(-n // 8) * 8
        return out

    def forward(self, tokens, drops):
        """Logits [T][V][B] of tokens [T][B] (int32)."""
        L.embed(tokens, self.E, scale=self.scale, drop=drops[0], out=self.inputs[0])
        for l in range(self.cfg.layers):
            L.fwd_cache(self.inputs[l], self.Ws[l], self.bs[l], h_out=self.houts[l], cache=self.caches[l],
                        ws=self.fws[l])
            nxt = self.inputs[l + 1] if l + 1 < self.cfg.layers else self.top
            if drops[l + 1] is not None:
                L.dropout(self.houts[l], drops[l + 1], out=nxt)
            else:
                nxt.copy_(self.houts[l])
        if self.head:
            return self._head(self.top, self.logits, self.act, self.head_ws)
        for t in range(self.cfg.steps):
            torch.mm(self.Wv, self.top[t], out=self.logits[t])
        return self.logits

    def backward(self, tokens, drops, sparse: bool):
        """Gradients of everything from dL/dlogits, which stands in the logits' place."""
        cfg, d = self.cfg, self.logits
        if self.head:
            self._head_backward()
        else:
            self.dWv.zero_()
            for t in range(cfg.steps):
                self.dH[t] = _product(self.Wv.t(), d[t])
                self.dWv += _product(d[t], self.top[t].t())
        up = self.dH
        for l in range(cfg.layers - 1, -1, -1):
            if drops[l + 1] is not None:
                L.dropout(up, drops[l + 1], out=up)
            call = dict(out=self.outs[l], ws=self.ws)
            self.outs[l] = L.bwd_structsparse(self.inputs[l], self.Ws[l], self.caches[l], up, sparsity=cfg.sparsity,
                                              P=cfg.P, R=cfg.R, want_idx=False, **call) if sparse else \
                L.bwd_dense(self.inputs[l], self.Ws[l], self.caches[l], up, **call)
            up = self.outs[l]["dX"]
        L.embed_grad(tokens, up, cfg.vocabulary, scale=self.scale, drop=drops[0], dE=self.dE, ws=self.dE_ws)

    def _muon(self, name, W, dW, blocks):
        if name not in self.moments:
            self.moments[name] = torch.zeros(W.shape, device=W.device)
        L.muon_update(W, self.moments[name], dW, self.cfg.muon_lr, momentum=self.cfg.momentum, blocks=blocks,
                      ws=self.muon_ws)

    def update(self):
        """SGD with a fixed learning rate; with optimizer "muon" orthogonalised momentum for the
        layers' weights (each gate by itself) and the block's."""
        lr, muon = self.cfg.lr, self.cfg.optimizer == "muon"
        for l in range(self.cfg.layers):
            o = self.outs[l]
            if muon:
                self._muon(l, self.Ws[l], o["dW"], 4)
                self.bs[l].sub_(o["db"], alpha=lr)
            else:
                L.sgd_update(self.Ws[l], self.bs[l], o["dW"], o["db"], lr, self.cfg.layer_input(l))
        self.E.copy_(self.E.float().sub_(self.dE, alpha=lr))
        self.Wv.copy_(self.Wv.float().sub_(self.dWv, alpha=lr))
        for name, w in self.head.items():
            if muon and w.dim() == 2:
                self._muon(name, w, self.grads[name], 1)
            else:
                w.copy_(w.float().sub_(self.grads[name], alpha=lr))

    def _loss_scale(self, targets):
        return 1.0 / (self.cfg.steps * self.cfg.batch)

    def step(self, tokens, targets, sparse: bool = False, update: bool = True):
        """One training step on targets [T][B] (int32, -1: none); returns the loss [1], the mean
        over T * B of the targets' -logp."""
        drops = self._drops(True)
        self.forward(tokens, drops)
        L.xent(self.logits, targets, scale=self._loss_scale(targets), out=self.loss_out, ws=self.loss_ws)
        self.backward(tokens, drops, sparse)
        if update:
            self.update()
        return self.loss_out["loss"]

    def score(self, tokens, targets):
        """The targets' log probabilities [T][B] without dropout (a new tensor)."""
        logits = self.forward(tokens, [None] * (self.cfg.layers + 1))
        return L.token_logp(logits, targets, ws=self.loss_ws)

    def generate(self, prompt, beams: int, steps: int, eos: int = -1):
        """Answers of `steps` tokens to prompts [T0][S] (int32, no padding) by beam search without
        dropout: dict(tokens [steps][S * beams], scores [S * beams]), a sequence's beams side by
        side, the best first; after its first eos an answer goes on with eos."""
        cfg, dev, K = self.cfg, prompt.device, int(beams)
        if prompt.dim() != 2 or steps < 1 or K < 1:
            raise ValueError("prompt must be [T0][S], steps and beams positive")
        S, H = prompt.shape[1], cfg.hidden
        N = S * K
        # the layers' h and c after the prompt, for every beam of its sequence
        x, ends = L.embed(prompt, self.E, scale=self.scale), []
        for l in range(cfg.layers):
            x, cache = L.fwd_cache(x, self.Ws[l], self.bs[l])
            _, c, h = L.cache_views(cache, x.shape[0], S, H, cfg.dtype)
            ends += [h[-1].float(), c[-1]]
        states = torch.stack(ends).repeat_interleave(K, 2)
        moved = torch.empty_like(states)
        top = x[-1:].contiguous()
        logits = self._head(top)[0].repeat_interleave(K, 1)
        scores = torch.where(torch.arange(N, device=dev) % K == 0, 0.0, -math.inf)
        out = {"scores": scores}
        if eos >= 0:
            out["done"] = torch.zeros(N, dtype=torch.int32, device=dev)
        tokens, parents = (torch.empty((steps, N), dtype=torch.int32, device=dev) for _ in range(2))
        ws = torch.empty(L.beam_workspace_bytes(S, K, cfg.vocabulary, cfg.dtype), dtype=torch.uint8, device=dev)
        for t in range(steps):
            out.update(tokens=tokens[t], parents=parents[t])
            L.beam_step(logits, scores, K, eos=eos, done=out.get("done"), out=out, ws=ws)
            if t + 1 == steps:
                break
            L.beam_reorder(states, parents[t], K, out=moved)
            states, moved = moved, states
            x = L.embed(tokens[t:t + 1], self.E, scale=self.scale)
            for l in range(cfg.layers):
                x, cache = L.fwd_cache(x, self.Ws[l], self.bs[l], h0=states[2 * l], c0=states[2 * l + 1])
                _, c, _ = L.cache_views(cache, 1, N, H, cfg.dtype)
                states[2 * l].copy_(x[0])
                states[2 * l + 1].copy_(c[1])
            logits = self._head(x)[0]
        return {"tokens": L.beam_trace(tokens, parents, K), "scores": scores}

    def policy_step(self, tokens, targets, old, ref, adv, clip_low=0.2, clip_high=0.2, kl=0.0,
                    sparse: bool = False, update: bool = True):
        """One step of the clipped policy loss: old and ref (may be None) are logp as score()
        gives them, adv the tokens' advantages, all [T][B]."""
        drops = self._drops(False)
        self.forward(tokens, drops)
        L.policy_loss(self.logits, targets, old, ref, adv, clip_low=clip_low, clip_high=clip_high, kl=kl,
                      scale=self._loss_scale(targets), out=self.loss_out, ws=self.loss_ws)
        self.backward(tokens, drops, sparse)
        if update:
            self.update()
        return self.loss_out["loss"]


def make_weights(cfg: LanguageConfig, device="cuda:0"):
    """Uniform weights of 0.1, zero biases, from cfg.seed."""
    g = torch.Generator().manual_seed(cfg.seed)

    def uniform(*shape):
        return ((torch.rand(shape, generator=g) - 0.5) * 0.2).to(device=device, dtype=cfg.dtype)

    H = cfg.hidden
    return (uniform(cfg.vocabulary, cfg.features),
            [uniform(4 * H, cfg.layer_input(l) + H) for l in range(cfg.layers)],
            [torch.zeros(4 * H, device=device) for _ in range(cfg.layers)],
            uniform(cfg.vocabulary, H))


def make_head(cfg: LanguageConfig, device="cuda:0"):
    """The head's weights besides Wv, uniform of 0.1, with zero biases, from cfg.seed + 1."""
    g = torch.Generator().manual_seed(cfg.seed + 1)
    return {k: torch.zeros(shape, device=device) if len(shape) == 1 else
            ((torch.rand(shape, generator=g) - 0.5) * 0.2).to(device=device, dtype=cfg.dtype)
            for k, shape in cfg.head_shapes().items()}


def synthetic_batch(cfg: LanguageConfig, seed: int, device="cuda:0"):
    """Tokens and next-token targets of sequences in which a token decides the next (5 times it
    and 3 more, modulo the vocabulary), half of them padded at the end."""
    g = torch.Generator().manual_seed(seed)
    T, B, V = cfg.steps, cfg.batch, cfg.vocabulary
    rows = [torch.randint(0, V, (B,), generator=g)]
    for _ in range(T):
        rows.append((5 * rows[-1] + 3) % V)
    s = torch.stack(rows)
    length = torch.where(torch.rand(B, generator=g) < 0.5, T, T - T // 4)
    s = torch.where(torch.arange(T + 1)[:, None] <= length[None, :], s, -1).to(torch.int32)
    return s[:-1].contiguous().to(device), s[1:].contiguous().to(device)


def main(steps: int = 60):
    from .train import dense_after_sparse
    cfg = LanguageConfig(vocabulary=200, features=64, hidden=128, layers=2, batch=32, steps=20, lr=4.0,
                         dropout=0.1)
    model = LanguageModel(cfg, *make_weights(cfg))
    losses = []
    for k, sparse in enumerate(dense_after_sparse(steps)):
        losses.append(float(model.step(*synthetic_batch(cfg, k), sparse=sparse)))
        if k % 10 == 0 or k == steps - 1:
            print("step %d (%s) loss %.4f" % (k, "sparse" if sparse else "dense", losses[-1]), flush=True)
    tokens, targets = synthetic_batch(cfg, 1000)
    before = model.score(tokens, targets)
    adv = torch.where(torch.arange(cfg.batch, device=tokens.device) % 2 == 0, 1.0, -1.0).expand(cfg.steps, -1)
    for _ in range(3):
        model.policy_step(tokens, targets, before, before, adv.contiguous(), kl=0.05)
    moved = (model.score(tokens, targets) - before).sum(0)
    print("policy update: logp of favoured sequences %+.3f, of the others %+.3f" %
          (float(moved[::2].mean()), float(moved[1::2].mean())), flush=True)
    answer(steps)
    return losses, moved


def answer(steps: int = 60, length: int = 8):
    """Trains a model with a residual block and orthogonalised momentum on the same sequences
    and lets it answer prompts of four tokens; returns the share of right tokens."""
    cfg = LanguageConfig(vocabulary=200, features=64, hidden=128, layers=2, batch=32, steps=20, lr=1.0,
                         dropout=0.1, head_bias=True, block=256, optimizer="muon")
    E, Ws, bs, Wv = make_weights(cfg)
    model = LanguageModel(cfg, E, Ws, bs, Wv, head=make_head(cfg))
    for k in range(steps):
        loss = model.step(*synthetic_batch(cfg, k))
    print("block and orthogonalised momentum: loss %.4f" % float(loss), flush=True)
    prompt = synthetic_batch(cfg, 1001)[0][:4].contiguous()
    out = model.generate(prompt, beams=4, steps=length)
    best, last = out["tokens"][:, ::4].long(), prompt[-1].long()
    right = []
    for t in range(length):
        last = (5 * last + 3) % cfg.vocabulary
        right.append(best[t] == last)
    share = float(torch.stack(right).float().mean())
    print("answers: %.0f %% of the best beams' tokens are right" % (100 * share), flush=True)
    return share


if __name__ == "__main__":
    main()
