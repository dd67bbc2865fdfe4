"""Tensors that the native checks leave to Python's, and that they do leave them:
the results are those of contiguous tensors, bit for bit."""
from __future__ import annotations

import pytest
import torch

import paper_2603_11438_amd as ar
from gpu_helpers import say
from paper_2603_11438_amd import ops

pytestmark = pytest.mark.gpu


class Wrapped(torch.Tensor):
    pass


def rand(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def sliced(rows, cols, seed):
    """2 x rows x cols, its rows at a stride: no matrix, not contiguous."""
    return rand(2, rows, cols + 24, seed=seed)[..., :cols]


def column(n, seed):
    """n x 1, strides (2, 96)."""
    return rand(96, 2 * n, seed=seed).t()[::2, :1]


OPERANDS = {
    "rows of a wider tensor": lambda seed: sliced(3, 96, seed),
    "a single column": lambda seed: column(5, seed),
    "a subclass": lambda seed: rand(6, 96, seed=seed).as_subclass(Wrapped),
}


@pytest.fixture
def answers(monkeypatch):
    """What the native functions answered, in order."""
    torch.cuda.init()
    nat = ops._native()
    assert nat is not None, "the native path is not built"
    got = []

    def spy(fn):
        def call(*a):
            got.append(fn(*a))
            return got[-1]
        return call

    for name in ("norm", "norm_backward", "ffn", "ffn_backward"):
        monkeypatch.setattr(nat, name, spy(getattr(nat, name)))
    return got


def plain(t):
    return torch.Tensor.contiguous(t.as_subclass(torch.Tensor)).clone()


def same(got, want):
    assert len(got) == len(want)
    for a, b in zip(got, want):
        assert torch.equal(a.as_subclass(torch.Tensor).reshape(b.shape), b)


@pytest.mark.parametrize("kind", list(OPERANDS))
def test_norm(answers, kind):
    say("fallback", kind)
    y, r, ds, dx = (OPERANDS[kind](seed) for seed in range(4))
    w = rand(y.shape[-1], seed=9)
    calls = (lambda y, r, ds, dx: ar.residual_norm(y, r, post_weight=w),
             lambda y, r, ds, dx: list(ar.residual_norm_backward(y, r, ds, dx, post_weight=w).values()))
    for call in calls:
        answers.clear()
        got = call(y, r, ds, dx)
        assert answers == [None], "the native checks took it"
        want = call(*(plain(t) for t in (y, r, ds, dx)))
        assert len(answers) == 2 and answers[1] is not None
        same(got, want)


@pytest.mark.parametrize("kind", ["rows of a wider tensor", "a subclass"])
def test_ffn(answers, kind):
    say("fallback ffn", kind)
    x, dh = OPERANDS[kind](0), OPERANDS[kind](1)[..., :40]
    wg, wu = rand(40, 96, seed=2), rand(40, 96, seed=3)
    answers.clear()
    h, saved = ar.gated_ffn(x, wg, wu, save=True)
    got = ar.gated_ffn_backward(dh, x, wg, wu, saved)
    assert answers == [None, None]
    want_h, want_saved = ar.gated_ffn(plain(x), wg, wu, save=True)
    want = ar.gated_ffn_backward(plain(dh), plain(x), wg, wu, want_saved)
    assert len(answers) == 4 and answers[2] is not None and answers[3] is not None
    same((h, saved, *got), (want_h, want_saved, *want))
