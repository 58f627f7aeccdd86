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
