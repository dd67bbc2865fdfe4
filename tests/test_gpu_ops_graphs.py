"""Results of the operators have no autograd graph, and a caller who would expect
one is told so, once."""
from __future__ import annotations

import warnings

import pytest
import torch

import paper_2603_11438_amd as ar
from gpu_helpers import say
from paper_2603_11438_amd import ops

pytestmark = pytest.mark.gpu


@pytest.fixture
def untold(monkeypatch):
    """As in a new process: a native path of its own, nothing told."""
    torch.cuda.init()
    monkeypatch.setattr(ops, "_native_path", None)
    monkeypatch.setattr(ops, "_graphs_told", False)
    return monkeypatch


def operands():
    g = torch.Generator().manual_seed(0)
    rnd = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731
    return rnd(6, 64), rnd(6, 64), rnd(40, 64), rnd(40, 64), rnd(64)


CALLS = {
    "residual_norm": lambda y, r, a, b, w: ar.residual_norm(y, r, post_weight=w)[0],
    "residual_norm_backward": lambda y, r, a, b, w: ar.residual_norm_backward(y, r, None, y, post_weight=w)["dpost_weight"],
    "gated_ffn": lambda y, r, a, b, w: ar.gated_ffn(y, a, b),
    "gated_ffn_backward": lambda y, r, a, b, w: ar.gated_ffn_backward(*_saved(y, a, b))[0],
    "orthogonalize": lambda y, r, a, b, w: ar.orthogonalize(a),
}


def _saved(y, a, b):
    with torch.no_grad():
        h, saved = ar.gated_ffn(y, a, b, save=True)
    return h, y, a, b, saved


@pytest.mark.parametrize("name", list(CALLS))
@pytest.mark.parametrize("native", (True, False))
def test_told_once(untold, name, native):
    say(f"graphs {name} native {native}")
    if not native:
        untold.setattr(ops, "_native_path", False)
    y, r, a, b, w = operands()
    want = CALLS[name](y, r, a, b, w)
    a.requires_grad_(), w.requires_grad_()
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with torch.no_grad():
            assert torch.equal(CALLS[name](y, r, a, b, w), want)
    with pytest.warns(RuntimeWarning, match="no autograd graph"):
        got = CALLS[name](y, r, a, b, w)
    assert torch.equal(got, want) and not got.requires_grad
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        got = CALLS[name](y, r, a, b, w)
    assert torch.equal(got, want) and not got.requires_grad
    assert "autograd" in ops.__doc__


def test_forward_mode_too(untold):
    y, r, *_ = operands()
    import torch.autograd.forward_ad as fwd

    with fwd.dual_level():
        s, x = ar.residual_norm(fwd.make_dual(y, r), r)
        assert fwd.unpack_dual(s).tangent is None and fwd.unpack_dual(x).tangent is None
