"""The vocabulary loss's requests that are refused before anything is launched, its
workspaces, and its plain form's gradients against differences (no GPU)."""
from __future__ import annotations

import ctypes
import os

import pytest
import torch

import paper_2603_11438_amd as ar
from oracle import ops_oracle as oo
from paper_2603_11438_amd import ops


@pytest.fixture(scope="module", autouse=True)
def built_lib():
    if not os.path.exists(ar.LIB_PATH):
        import __graft_entry__

        __graft_entry__.build()


# Addresses that are checked and never followed: every call below is refused.
X, W, T, LOSS, LSE, DLOSS, DX, DW, WS, PARTS = (0x10000000 * k for k in range(1, 11))


def desc(**kw):
    f = dict(tokens=16, dim=64, rows=100, first=0, classes=100, dtype=1, target_bytes=8)
    return ops.ar_vocab_desc(**{**f, **kw})


def forward(x=X, w=W, target=T, loss=LOSS, lse=LSE, ws=WS, nbytes=1 << 27, **kw):
    return ops._lib().ar_vocab_loss(ctypes.byref(desc(**kw)), x, w, target, loss, lse, ws, nbytes, None)


BAD_DESC = [
    (dict(dtype=0), ar.AR_ERR_UNSUPPORTED), (dict(target_bytes=2), ar.AR_ERR_UNSUPPORTED), (dict(dim=0), ar.AR_ERR_ARG),
    (dict(rows=0), ar.AR_ERR_ARG), (dict(dim=(1 << 20) + 1), ar.AR_ERR_ARG), (dict(rows=(1 << 26) + 1, classes=1 << 29), ar.AR_ERR_ARG),
    (dict(tokens=1 << 31), ar.AR_ERR_ARG), (dict(tokens=1 << 20, rows=1 << 20, classes=1 << 20), ar.AR_ERR_ARG), (dict(tokens=(1 << 24) + 1), ar.AR_ERR_ARG), (dict(first=1), ar.AR_ERR_ARG),
    (dict(first=1 << 60), ar.AR_ERR_ARG), (dict(classes=99), ar.AR_ERR_ARG), (dict(classes=1 << 50), ar.AR_ERR_ARG), (dict(ld_x=63), ar.AR_ERR_ARG),
    (dict(ld_w=1 << 50), ar.AR_ERR_ARG)]
BAD = BAD_DESC + [
    (dict(x=None), ar.AR_ERR_ARG), (dict(w=W + 1), ar.AR_ERR_ARG), (dict(target=None), ar.AR_ERR_ARG), (dict(target=T + 4), ar.AR_ERR_ARG),
    (dict(lse=None), ar.AR_ERR_ARG), (dict(lse=LSE + 2), ar.AR_ERR_ARG), (dict(ws=None), ar.AR_ERR_SCRATCH), (dict(nbytes=16), ar.AR_ERR_SCRATCH),
    (dict(ws=WS + 64), ar.AR_ERR_ARG), (dict(ws=X), ar.AR_ERR_ARG), (dict(ws=LSE), ar.AR_ERR_ARG)]


@pytest.mark.parametrize("kw,code", BAD + [
    (dict(loss=None), ar.AR_ERR_ARG), (dict(classes=200), ar.AR_ERR_ARG), (dict(loss=LSE), ar.AR_ERR_ARG), (dict(loss=W), ar.AR_ERR_ARG),
    (dict(lse=T), ar.AR_ERR_ARG)])
def test_forward_refusals(kw, code):
    assert forward(**kw) == code
    assert ar.ar_last_error() == code


@pytest.mark.parametrize("kw,code", [(dict(ranks=0), ar.AR_ERR_ARG), (dict(ranks=1 << 17), ar.AR_ERR_ARG), (dict(parts=None), ar.AR_ERR_ARG),
                                     (dict(loss=None), ar.AR_ERR_ARG), (dict(lse=LOSS), ar.AR_ERR_ARG), (dict(loss=PARTS + 64), ar.AR_ERR_ARG),
                                     (dict(target=T + 1), ar.AR_ERR_ARG), (dict(dtype=5), ar.AR_ERR_UNSUPPORTED)])
def test_join_refusals(kw, code):
    kw = dict(kw)
    a = {k: kw.pop(k, v) for k, v in dict(ranks=2, parts=PARTS, target=T, loss=LOSS, lse=LSE).items()}
    assert ops._lib().ar_vocab_loss_join(ctypes.byref(desc(**kw)), a["ranks"], a["parts"], a["target"], a["loss"], a["lse"], None) == code


def backward(dloss=DLOSS, stride=1, x=X, w=W, target=T, lse=LSE, dx=DX, dw=DW, ws=WS, nbytes=1 << 27, **kw):
    return ops._lib().ar_vocab_loss_backward(ctypes.byref(desc(**kw)), dloss, stride, x, w, target, lse, dx, dw, ws, nbytes, None)


@pytest.mark.parametrize("kw,code", BAD + [
    (dict(dloss=None), ar.AR_ERR_ARG), (dict(dloss=DLOSS + 2), ar.AR_ERR_ARG), (dict(stride=1 << 60), ar.AR_ERR_ARG), (dict(dx=DW), ar.AR_ERR_ARG),
    (dict(dx=X), ar.AR_ERR_ARG), (dict(dw=W), ar.AR_ERR_ARG), (dict(dw=LSE), ar.AR_ERR_ARG), (dict(dx=DX + 1), ar.AR_ERR_ARG),
    (dict(dx=WS), ar.AR_ERR_ARG), (dict(ld_dx=60), ar.AR_ERR_ARG), (dict(ld_dw=63), ar.AR_ERR_ARG)])
def test_backward_refusals(kw, code):
    assert backward(**kw) == code


def test_nothing_to_do():
    assert forward(tokens=0, x=None, ws=None) == ar.AR_OK
    assert backward(tokens=0, dw=None, x=None, ws=None) == ar.AR_OK
    assert backward(dx=None, dw=None, ws=None) == ar.AR_OK


def space(dx=1, dw=1, x=X, w=W, **kw):
    return ops._lib().ar_vocab_loss_backward_workspace(ctypes.byref(desc(**kw)), x, w, dx, dw)


def test_workspaces():
    """dz of a piece at a time; copies only of what cannot be read where it lies."""
    big = dict(tokens=4096, dim=4096, rows=131072, classes=131072)
    assert space(**big) <= (1 << 29) + 4096 * 4096 * 4 + 4096
    assert space(w=W + 2, **big) - space(**big) >= 131072 * 4096 * 2
    assert space(dx=0, dw=1, **big) < space(**big)
    assert ops._lib().ar_vocab_loss_workspace(ctypes.byref(desc(**big)), X, W) < 1 << 26
    for tokens in (1, 3, 64, 65, 1000, 40000, 300000):
        for rows in (1, 100, 1024, 5001, 131072):
            n = space(tokens=tokens, rows=rows, classes=rows, dim=256)
            assert n >= min(rows, 1024) * tokens * 2
            assert n <= max(1 << 29, tokens * 2 * 1024) + 33 * 4 * 256 * (tokens + rows) + (1 << 20)


def test_tensor_checks():
    t, w, target = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(5, 8, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: ar.vocab_loss(t, w, target), lambda: ar.vocab_loss_part(t, w, target, first=0),
                 lambda: ar.vocab_loss_join(torch.zeros(1, 2, 4), target, classes=5),
                 lambda: ar.vocab_loss_backward(torch.zeros(4), t, w, target, torch.zeros(4))):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_plain_gradient_is_the_difference():
    torch.manual_seed(3)
    rnd = lambda *s: torch.randn(*s, dtype=torch.float64)  # noqa: E731
    v, target, dloss, step = {"x": rnd(9, 6), "w": rnd(11, 6)}, torch.tensor([0, 10, -1, 3, 3, 11, -100, 5, 7]), rnd(9), 1e-6
    loss = lambda u: float((dloss * oo.vocab_loss(u["x"], u["w"], target)["loss"][0]).sum())  # noqa: E731
    grads = oo.vocab_loss(v["x"], v["w"], target, dloss)
    for name in v:
        e = rnd(*v[name].shape)
        fd = (loss({**v, name: v[name] + step * e}) - loss({**v, name: v[name] - step * e})) / (2 * step)
        assert abs(fd - float((grads["d" + name][0] * e).sum())) < 1e-6 * (1 + abs(fd)), name
