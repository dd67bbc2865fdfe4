"""Both ways into the operators, native checks and checks in Python, make the
same calls: results are compared bit for bit, refusals by their type."""
from __future__ import annotations

import pytest
import torch

import paper_2603_11438_amd as ar
from gpu_helpers import say
from paper_2603_11438_amd import ops

pytestmark = pytest.mark.gpu


def rand(*shape, dtype=torch.bfloat16, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def flat(got):
    if isinstance(got, dict):
        return [got[k] for k in sorted(got)]
    return list(got) if isinstance(got, tuple) else [got]


def both(monkeypatch, call):
    """The results of a call by the native checks (which must take it) and by Python's."""
    torch.cuda.init()
    nat = ops._native()
    assert nat is not None, "the native path is not built"
    first = flat(call())
    with monkeypatch.context() as m:
        m.setattr(ops, "_native_path", False)
        second = flat(call())
    assert len(first) == len(second)
    for a, b in zip(first, second):
        assert (a is None) == (b is None)
        if a is not None:
            assert a.shape == b.shape and a.dtype == b.dtype and a.stride() == b.stride() and torch.equal(a, b)


class Wrapped(torch.Tensor):
    pass


NORMS = [dict(), dict(post_weight=1), dict(post_weight=1, pre_weight=1, gate=1, alpha=0.5), dict(gate=2), dict(post=False, pre_weight=1),
         dict(pre=False, post_weight=1)]


@pytest.mark.parametrize("which", range(len(NORMS)))
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm(monkeypatch, which, dtype):
    kw = dict(NORMS[which])
    rows, cols = 6, 200
    if "gate" in kw:
        kw["gate"] = rand(cols, seed=3, dtype=dtype) if kw["gate"] == 1 else rand(2, cols, seed=3, dtype=dtype)
    for k in ("post_weight", "pre_weight"):
        if k in kw:
            kw[k] = rand(cols, seed=4, dtype=dtype)
    y, r = rand(2, 3, cols, dtype=dtype), rand(2, 3, cols, seed=1, dtype=dtype)
    say("norm", which, dtype)
    both(monkeypatch, lambda: ar.residual_norm(y, r, **kw))
    s, x = ar.residual_norm(y, r, **kw)
    dx = None if x is None else rand(2, 3, cols, seed=5, dtype=dtype)
    both(monkeypatch, lambda: ar.residual_norm_backward(y, s, rand(2, 3, cols, seed=6, dtype=dtype), dx, **kw))
    wide = rand(rows, cols + 24, dtype=dtype)[:, :cols]  # rows at a stride
    both(monkeypatch, lambda: ar.residual_norm(wide, r.view(rows, cols), **kw))


@pytest.mark.parametrize("tokens,dim,hidden", [(1, 64, 40), (5, 72, 130), (70, 100, 65)])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_ffn(monkeypatch, tokens, dim, hidden, act):
    say("ffn", tokens, dim, hidden, act)
    x, w = rand(tokens, dim), rand(2 * hidden, dim, seed=1)
    wg, wu = w[:hidden], w[hidden:]  # halves of one tensor
    both(monkeypatch, lambda: ar.gated_ffn(x, wg, wu, act=act))
    both(monkeypatch, lambda: ar.gated_ffn(x, wg, wu, act=act, save=True))
    h, saved = ar.gated_ffn(x, wg, wu, act=act, save=True)
    for need in (dict(), dict(need_dx=False), dict(need_dw=False)):
        both(monkeypatch, lambda: ar.gated_ffn_backward(h, x, wg, wu, saved, act=act, **need))


def test_left_to_python():
    """What the native checks do not take gives the same results by way of Python's."""
    y, r = rand(4, 96), rand(4, 96, seed=1)
    want = ar.residual_norm(y, r)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = [ar.residual_norm(y.as_subclass(Wrapped), r), ar.residual_norm(y.t().contiguous().t().contiguous(), r),
           ar.residual_norm(y, r, out=(torch.empty_like(y), torch.empty_like(y))), ar.residual_norm(y, r, stream=other)]
    torch.cuda.synchronize()
    for s, x in got:
        assert torch.equal(s, want[0]) and torch.equal(x, want[1])
    with torch.cuda.stream(other):
        s, x = ar.residual_norm(y, r)  # native, on the current stream
    other.synchronize()
    assert torch.equal(s, want[0]) and torch.equal(x, want[1])


BAD = {
    "another length": lambda y: ar.residual_norm(y, y[:, :-8]),
    "another type": lambda y: ar.residual_norm(y, y.float()),
    "on the CPU": lambda y: ar.residual_norm(y, y.cpu()),
    "a double": lambda y: ar.residual_norm(y.double(), y.double()),
    "columns apart": lambda y: ar.residual_norm(y.t(), y.t()),
    "a weight's length": lambda y: ar.residual_norm(y, y, post_weight=y[0, :-1]),
    "a weight that is not used": lambda y: ar.residual_norm(y, y, post_weight=y[0], post=False),
    "gate rows": lambda y: ar.residual_norm(y, y, gate=y[:3]),
    "eps": lambda y: ar.residual_norm(y, y, eps=-1.0),
    "an activation": lambda y: ar.gated_ffn(y, y, y, act="tanh"),
    "fp32 operands": lambda y: ar.gated_ffn(y.float(), y.float(), y.float()),
    "weights' shapes": lambda y: ar.gated_ffn(y, y, y[:2]),
    "saved": lambda y: ar.gated_ffn_backward(y[:, :4], y, y[:4], y[:4], y),
}


@pytest.mark.parametrize("what", list(BAD))
def test_refused_alike(monkeypatch, what):
    y = rand(4, 96)
    say("refused", what)
    kinds = []
    for path in (None, False):
        with monkeypatch.context() as m:
            if path is False:
                m.setattr(ops, "_native_path", False)
            with pytest.raises((ValueError, TypeError, ar.ARError)) as e:
                BAD[what](y)
            kinds.append(e.type)
    assert kinds[0] is kinds[1]
