"""CPU: whose memory a call on another stream works on.

The allocator gives a block that was freed on a stream out again on that stream
at once, while kernels there may still be at work on it.  So what a call on a
given stream allocates has to come from that stream's own blocks, and what it
hands back has to be known on the caller's.  Here the allocator and the library
stand in for the real ones and note what is asked of them."""
import contextlib
import types

import pytest
import torch

import paper_1806_00512_amd.lstmss as L

F32, I32, U8 = torch.float32, torch.int32, torch.uint8


class Made(torch.Tensor):
    """A tensor that notes the stream it was made on and those it is said to be used on."""

    def record_stream(self, stream):
        self.used_on.append(stream.name)


class Lib:
    """Every size is 64 bytes (or entries), every call succeeds."""

    def __getattr__(self, name):
        size = name.endswith(("_bytes", "_rows", "_entries"))
        return lambda *args: 64 if size else 0


@pytest.fixture
def made(monkeypatch):
    def stream(name):
        return types.SimpleNamespace(name=name, device=torch.device("cuda", 0), cuda_stream=1)

    now, out, real = [stream("caller")], [], torch.empty

    def empty(*shape, dtype=None, device=None):
        t = real(*shape, dtype=dtype).as_subclass(Made)
        t.made_on, t.used_on = now[-1].name, []
        out.append(t)
        return t

    @contextlib.contextmanager
    def on(s):
        now.append(s)
        yield
        now.pop()

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch, "empty_like", lambda t: empty(tuple(t.shape), dtype=t.dtype))
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: now[-1])
    monkeypatch.setattr(L, "load", Lib)
    monkeypatch.setattr(L, "_on", lambda first, name, s: (0, 1))
    for name in ("_at", "_ptr"):
        monkeypatch.setattr(L, name, lambda *a, **k: None)
    return types.SimpleNamespace(all=out, side=stream("side"))


def z(*shape, dtype=F32):
    return torch.zeros(shape, dtype=dtype)


LANGUAGE = {
    "dropout": lambda s: L.dropout(z(4, 5), L.drop(0.5, 1), stream=s),
    "embed": lambda s: L.embed(z(2, 3, dtype=I32), z(7, 4), stream=s),
    "embed_grad": lambda s: L.embed_grad(z(2, 3, dtype=I32), z(2, 4, 3), 7, stream=s),
    "token_logp": lambda s: L.token_logp(z(2, 7, 3), z(2, 3, dtype=I32), stream=s),
    "xent": lambda s: L.xent(z(2, 7, 3), z(2, 3, dtype=I32), stream=s),
    "policy_loss": lambda s: L.policy_loss(z(2, 7, 3), z(2, 3, dtype=I32), None, None, z(2, 3), stream=s),
}


def check(call, made):
    call(made.side)
    assert made.all and all(t.made_on == "side" for t in made.all)
    assert all("caller" in t.used_on for t in made.all)
    del made.all[:]
    call(None)
    assert made.all and all(t.made_on == "caller" and not t.used_on for t in made.all)


@pytest.mark.parametrize("name", LANGUAGE)
def test_language_calls(made, name):
    check(LANGUAGE[name], made)


def layer(T=2, B=3, I=4, H=8):
    return z(T, I, B), z(4 * H, I + H), z(64, dtype=U8), z(T, H, B)


def bidirectional(s):
    x, W, cache, _ = layer()
    return L.bwd_bidir(x, x, W, W, cache, cache, z(2, 16, 3), stream=s)


LAYERS = {
    "fwd_cache": lambda s: L.fwd_cache(*layer()[:2], stream=s),
    "mse_grad": lambda s: L.mse_grad(z(2, 8, 3), z(2, 8, 3), stream=s),
    "bwd_dense": lambda s: L.bwd_dense(*layer(), stream=s),
    "bwd_structsparse": lambda s: L.bwd_structsparse(*layer(), want_dbg=True, stream=s),
    "bwd_stack": lambda s: L.bwd_stack(*[[a] for a in layer()[:3]], layer()[3], want_dX0=True, stream=s),
    "bwd_bidir": bidirectional,
    "time_reverse": lambda s: L.time_reverse(z(2, 4, 3), stream=s),
    "bidir_join": lambda s: L.bidir_join(z(2, 8, 3), z(2, 8, 3), stream=s),
    "select_compact": lambda s: L.select_compact(z(32, 3), stream=s),
    "select_compact_fine": lambda s: L.select_compact(z(32, 3), kind=L.FINE, My=8, Mx=4, stream=s),
}


@pytest.mark.parametrize("name", LAYERS)
def test_layer_calls(made, name):
    check(LAYERS[name], made)


@pytest.mark.gpu
def test_layer_results_on_another_stream():
    """Forward and backward of a layer on a given stream, all buffers the calls' own: the bits
    of the current stream's calls, in memory that is not the current stream's."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    T, B, I, H = 5, 20, 40, 72
    g = torch.Generator().manual_seed(0)
    x, W, up = (torch.randn(s, generator=g).cuda() * 0.1 for s in ((T, I, B), (4 * H, I + H), (T, H, B)))

    def calls(stream):
        h, cache = L.fwd_cache(x, W, stream=stream)
        return h, L.bwd_structsparse(x, W, cache, up, stream=stream)

    h, want = calls(None)
    torch.cuda.synchronize()
    freed = torch.empty_like(h)
    at = freed.data_ptr()
    del freed
    side = torch.cuda.Stream()
    h2, got = calls(side)
    side.synchronize()
    assert h2.data_ptr() != at and torch.equal(h2, h)
    assert all(torch.equal(got[k], want[k]) for k in want if want[k] is not None)
