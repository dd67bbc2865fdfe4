"""Both ways into attention and the vocabulary loss, native checks and checks in Python,
make the same calls: results are compared bit for bit, refusals by their type; and
callers are told that results have no autograd graph."""
from __future__ import annotations

import warnings

import pytest
import torch

import paper_2603_11438_amd as ar
from gpu_helpers import say
from paper_2603_11438_amd import ops

pytestmark = pytest.mark.gpu


def rand(*shape, dtype=torch.bfloat16, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def both(monkeypatch, call):
    torch.cuda.init()
    nat = ops._native()
    assert nat is not None, "the native path is not built"
    taken = []
    with monkeypatch.context() as m:
        for name in ("attention", "vocab_loss"):
            f = getattr(nat, name)
            m.setattr(nat, name, lambda *a, f=f: taken.append(f(*a)) or taken[-1])
        first = call()
    assert len(taken) == 1 and taken[0] is not None, "not taken by the native checks"
    with monkeypatch.context() as m:
        m.setattr(ops, "_native_path", False)
        second = call()
    for a, b in zip(first if isinstance(first, tuple) else [first], second if isinstance(second, tuple) else [second]):
        assert a.shape == b.shape and a.dtype == b.dtype and a.stride() == b.stride() and torch.equal(a, b)


@pytest.mark.parametrize("dim", [64, 100])
@pytest.mark.parametrize("save", [True, False])
def test_attention(monkeypatch, dim, save):
    say("attention", dim, save)
    qkv = rand(50, 8, dim)
    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    at = torch.tensor([0, 20, 45], dtype=torch.int32).cuda()
    keys = torch.tensor([0, 30, 50], dtype=torch.int32).cuda()
    for kw in (dict(), dict(starts_q=at), dict(starts_q=at, starts_k=keys, causal=False), dict(scale=0.3), dict(scale=1)):
        both(monkeypatch, lambda: ar.packed_attention(q, k, v, save=save, **kw))
    heads_first = rand(4, 50, dim).transpose(0, 1)
    both(monkeypatch, lambda: ar.packed_attention(heads_first, k, v, save=save))
    both(monkeypatch, lambda: ar.packed_attention(q[:1], k[:, :1], v[:, :1], save=save))


@pytest.mark.parametrize("kind", [torch.int64, torch.int32])
@pytest.mark.parametrize("dim", [64, 70])
def test_vocab_loss(monkeypatch, kind, dim):
    say("loss", kind, dim)
    x, w, t = rand(6, 5, dim), rand(200, dim + 6)[:, :dim], torch.arange(-3, 27).to(kind).cuda()
    both(monkeypatch, lambda: ar.vocab_loss(x, w, t.view(6, 5)))
    both(monkeypatch, lambda: ar.vocab_loss(x.view(30, dim)[:1], w, t[3:4]))


def test_on_the_stream_of_the_caller():
    q, k, v = rand(50, 4, 64), rand(50, 2, 64, seed=1), rand(50, 2, 64, seed=2)
    x, t = rand(30, 64), torch.arange(30).cuda()
    want = ar.packed_attention(q, k, v), *ar.vocab_loss(x, q[:, 0], t)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        got = ar.packed_attention(q, k, v), *ar.vocab_loss(x, q[:, 0], t)
    other.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


CALLS = {
    "attention": lambda q, x, t: ar.packed_attention(q, q, q),
    "attention backward": lambda q, x, t: ar.packed_attention_backward(q, q, q, q, q, torch.zeros(2, 9, device="cuda"))[0],
    "loss": lambda q, x, t: ar.vocab_loss(x, q[:, 0], t)[0],
    "loss part": lambda q, x, t: ar.vocab_loss_part(x, q[:, 0], t, first=0),
    "loss backward": lambda q, x, t: ar.vocab_loss_backward(torch.ones(4, device="cuda"), x, q[:, 0], t, torch.zeros(4, device="cuda"))[0],
}


@pytest.mark.parametrize("name", list(CALLS))
@pytest.mark.parametrize("native", (True, False))
def test_told_that_there_is_no_graph(monkeypatch, name, native):
    torch.cuda.init()
    monkeypatch.setattr(ops, "_native_path", None if native else False)
    monkeypatch.setattr(ops, "_graphs_told", False)
    q, x, t = rand(9, 2, 64), rand(4, 64), torch.arange(4).cuda()
    want = CALLS[name](q, x, t)
    q.requires_grad_(), x.requires_grad_()
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with torch.no_grad():
            assert torch.equal(CALLS[name](q, x, t), want)
    with pytest.warns(RuntimeWarning, match="no autograd graph"):
        got = CALLS[name](q, x, t)
    assert torch.equal(got, want) and not got.requires_grad
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        CALLS[name](q, x, t)


class Wrapped(torch.Tensor):
    pass


def test_left_to_python():
    q = rand(9, 2, 64)
    want = ar.packed_attention(q, q, q)
    assert torch.equal(ar.packed_attention(q.as_subclass(Wrapped), q, q).as_subclass(torch.Tensor), want)
    assert torch.equal(ar.packed_attention(q, q, q, out=torch.empty_like(q)), want)


BAD = {
    "fp32": lambda q, x, t: ar.packed_attention(q.float(), q.float(), q.float()),
    "heads": lambda q, x, t: ar.packed_attention(q[:, :1], q, q),
    "keys and values": lambda q, x, t: ar.packed_attention(q, q, q[:5]),
    "dim": lambda q, x, t: ar.packed_attention(q, q[..., :32], q[..., :32]),
    "starts": lambda q, x, t: ar.packed_attention(q, q, q, starts_q=t),
    "keys' starts alone": lambda q, x, t: ar.packed_attention(q, q, q, starts_k=t.int()),
    "scale": lambda q, x, t: ar.packed_attention(q, q, q, scale=-1.0),
    "scale's type": lambda q, x, t: ar.packed_attention(q, q, q, scale="1"),
    "overlapping heads": lambda q, x, t: ar.packed_attention(q, q[:, :1].expand(9, 2, 64), q),
    "target's length": lambda q, x, t: ar.vocab_loss(x, q[:, 0], t[:3]),
    "target's type": lambda q, x, t: ar.vocab_loss(x, q[:, 0], t.float()),
    "weight's width": lambda q, x, t: ar.vocab_loss(x, q[:, 0, :32], t),
    "weight's type": lambda q, x, t: ar.vocab_loss(x, q[:, 0].float(), t),
    "weight's shape": lambda q, x, t: ar.vocab_loss(x, q, t),
    "loss in fp32": lambda q, x, t: ar.vocab_loss(x.float(), q[:, 0].float(), t),
}


@pytest.mark.parametrize("what", list(BAD))
def test_refused_alike(monkeypatch, what):
    q, x, t = rand(9, 2, 64), rand(4, 64), torch.arange(4).cuda()
    say("refused", what)
    kinds = []
    for path in (None, False):
        with monkeypatch.context() as m:
            if path is False:
                m.setattr(ops, "_native_path", False)
            with pytest.raises((ValueError, TypeError, ar.ARError)) as e:
                BAD[what](q, x, t)
            kinds.append(e.type)
    assert kinds[0] is kinds[1]
