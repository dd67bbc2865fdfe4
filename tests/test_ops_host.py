"""Host-side checks of the operators around the collectives that need no GPU:
every call of include/ar_ops.h is exported and bound, wrong requests are
refused before anything is launched, and the plain forms' gradients agree with
differences."""
from __future__ import annotations

import ctypes
import os
import re

import pytest
import torch

import paper_2603_11438_amd as ar
from oracle import ops_oracle as oo
from paper_2603_11438_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def built_lib():
    if not os.path.exists(ar.LIB_PATH):
        import __graft_entry__

        __graft_entry__.build()
    ops._lib()


def test_every_declared_symbol_is_exported():
    text = open(os.path.join(ROOT, "include", "ar_ops.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(ar_[a-z0-9_]+)\s*\(", text))
    L = ctypes.CDLL(ar.LIB_PATH)
    assert names == set(ops.SIGNATURES)
    for n in names:
        assert hasattr(L, n), n


# Addresses that are checked and never followed: every call below is refused.
A, B, C, D = (0x10000000 * k for k in range(1, 5))


def norm(s=C, x=D, y=A, residual=B, w1=None, gate=None, w2=None, **kw):
    f = dict(rows=4, cols=64, dtype=0, param_dtype=0, flags=3, alpha=1.0, eps=1e-6)
    f.update(kw)
    return ops._lib().ar_residual_norm(ctypes.byref(ops.ar_norm_desc(**f)), y, residual, w1, gate, w2, s, x, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), ar.AR_ERR_UNSUPPORTED), (dict(param_dtype=-1), ar.AR_ERR_UNSUPPORTED), (dict(cols=0), ar.AR_ERR_ARG),
    (dict(flags=4), ar.AR_ERR_ARG), (dict(eps=0.0), ar.AR_ERR_ARG), (dict(eps=float("nan")), ar.AR_ERR_ARG),
    (dict(alpha=float("inf")), ar.AR_ERR_ARG), (dict(gate_rows=3, gate=0x90000000), ar.AR_ERR_ARG),
    (dict(gate_rows=2), ar.AR_ERR_ARG), (dict(ld_y=63), ar.AR_ERR_ARG), (dict(y=None), ar.AR_ERR_ARG),
    (dict(x=None), ar.AR_ERR_ARG), (dict(s=C + 2), ar.AR_ERR_ARG), (dict(s=A + 4), ar.AR_ERR_ARG), (dict(x=C), ar.AR_ERR_ARG),
    (dict(x=A, ld_x=65), ar.AR_ERR_ARG), (dict(w2=C + 64), ar.AR_ERR_ARG), (dict(rows=1 << 60), ar.AR_ERR_ARG)])
def test_norm_refusals(kw, code):
    assert norm(**kw) == code
    assert ar.ar_last_error() == code


def test_norm_without_rows_is_done():
    assert norm(rows=0, y=None, s=None, x=None, residual=None) == ar.AR_OK


def norm_bwd(ws=0xE0000000, nbytes=None, y=A, s=B, ds=None, dx=C, w1=None, gate=None, w2=None, dy=D, dr=0x50000000,
             dw1=None, dgate=None, dw2=None, **kw):
    f = dict(rows=4, cols=64, dtype=0, param_dtype=0, flags=3, alpha=1.0, eps=1e-6)
    f.update(kw)
    d = ops.ar_norm_desc(**f)
    L = ops._lib()
    n = L.ar_residual_norm_backward_workspace(ctypes.byref(d)) if nbytes is None else nbytes
    return L.ar_residual_norm_backward(ctypes.byref(d), y, s, ds, dx, w1, gate, w2, dy, dr, dw1, dgate, dw2, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dx=None), ar.AR_ERR_ARG), (dict(dw1=0x60000000, flags=2), ar.AR_ERR_ARG), (dict(dw2=0x60000000, flags=1), ar.AR_ERR_ARG),
    (dict(dgate=0x60000000), ar.AR_ERR_ARG), (dict(dw1=0x60000000, nbytes=8), ar.AR_ERR_SCRATCH),
    (dict(dw1=0x60000000, ws=None), ar.AR_ERR_SCRATCH), (dict(dw1=0x60000000, ws=0xE0000010), ar.AR_ERR_ARG),
    (dict(dw1=0x60000000, dw2=0x60000080), ar.AR_ERR_ARG), (dict(dw1=A), ar.AR_ERR_ARG), (dict(dy=A + 16), ar.AR_ERR_ARG),
    (dict(dr=D), ar.AR_ERR_ARG), (dict(dw1=0xE0000000), ar.AR_ERR_ARG)])
def test_norm_backward_refusals(kw, code):
    assert norm_bwd(**kw) == code


def test_norm_tensor_checks():
    """CPU tensors never reach the library."""
    t = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU"):
        ar.residual_norm(t, t)
    with pytest.raises(ValueError, match="GPU"):
        ar.residual_norm_backward(t, t, t, t)


def test_norm_plain_gradient_is_the_difference():
    torch.manual_seed(0)
    t, d, h = 6, 16, 1e-5
    rnd = lambda *s: torch.randn(*s, dtype=torch.float64)  # noqa: E731
    v = dict(y=rnd(t, d), residual=rnd(t, d), w1=rnd(d), w2=rnd(d), gate=rnd(3, d))
    ds, dx = rnd(t, d), rnd(t, d)

    def loss(**u):
        s, x, _, _ = oo.residual_norm(u["y"], u["residual"], u["w1"], u["w2"], u["gate"], 0.7, 1e-3)
        return float((s * ds).sum() + (x * dx).sum())

    s = oo.residual_norm(v["y"], v["residual"], v["w1"], v["w2"], v["gate"], 0.7, 1e-3)[0]
    g = oo.residual_norm_backward(v["y"], s, ds, dx, v["w1"], v["w2"], v["gate"], 0.7, 1e-3)
    for name, key in {"y": "dy", "residual": "dresidual", "w1": "dpost_weight", "w2": "dpre_weight", "gate": "dgate"}.items():
        e = rnd(*v[name].shape)
        fd = (loss(**{**v, name: v[name] + h * e}) - loss(**{**v, name: v[name] - h * e})) / (2 * h)
        assert abs(fd - float((g[key][0] * e).sum())) < 1e-6 * (1 + abs(fd)), name


def ffn(x=A, wg=B, wu=C, h=D, saved=None, ws=None, nbytes=0, **kw):
    f = dict(tokens=4, dim=64, hidden=32, dtype=1, act=0)
    f.update(kw)
    return ops._lib().ar_gated_ffn(ctypes.byref(ops.ar_ffn_desc(**f)), x, wg, wu, h, saved, ws, nbytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=0), ar.AR_ERR_UNSUPPORTED), (dict(dtype=7), ar.AR_ERR_UNSUPPORTED), (dict(act=3), ar.AR_ERR_ARG),
    (dict(dim=0), ar.AR_ERR_ARG), (dict(hidden=0), ar.AR_ERR_ARG), (dict(tokens=1 << 31), ar.AR_ERR_ARG),
    (dict(ld_x=60), ar.AR_ERR_ARG), (dict(ld_h=31), ar.AR_ERR_ARG), (dict(x=None), ar.AR_ERR_ARG), (dict(wu=C + 1), ar.AR_ERR_ARG),
    (dict(h=A), ar.AR_ERR_ARG), (dict(h=C + 2), ar.AR_ERR_ARG), (dict(saved=0x90000004), ar.AR_ERR_ARG), (dict(saved=A), ar.AR_ERR_ARG),
    (dict(saved=D), ar.AR_ERR_ARG), (dict(dim=60), ar.AR_ERR_SCRATCH), (dict(x=A + 2), ar.AR_ERR_SCRATCH),
    (dict(ld_w_up=65), ar.AR_ERR_SCRATCH), (dict(dim=60, ws=0x90000000, nbytes=100), ar.AR_ERR_SCRATCH),
    (dict(dim=60, ws=0x90000008, nbytes=1 << 20), ar.AR_ERR_ARG), (dict(dim=60, ws=A, nbytes=1 << 20), ar.AR_ERR_ARG)])
def test_ffn_refusals(kw, code):
    assert ffn(**kw) == code
    assert ar.ar_last_error() == code


def ffn_bwd(dh=A, x=B, wg=C, wu=D, saved=0x50000000, dx=0x60000000, dwg=0x70000000, dwu=0x80000000, ws=0x90000000,
            nbytes=None, **kw):
    f = dict(tokens=4, dim=64, hidden=32, dtype=1, act=0)
    f.update(kw)
    d = ops.ar_ffn_desc(**f)
    L = ops._lib()
    n = L.ar_gated_ffn_backward_workspace(ctypes.byref(d)) if nbytes is None else nbytes
    return L.ar_gated_ffn_backward(ctypes.byref(d), dh, x, wg, wu, saved, dx, dwg, dwu, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(saved=None), ar.AR_ERR_ARG), (dict(dwg=None), ar.AR_ERR_ARG), (dict(ws=None), ar.AR_ERR_SCRATCH),
    (dict(nbytes=1024), ar.AR_ERR_SCRATCH), (dict(ws=0x90000010), ar.AR_ERR_ARG), (dict(dx=B), ar.AR_ERR_ARG),
    (dict(dwg=0x80000800), ar.AR_ERR_ARG), (dict(dx=0x90000000), ar.AR_ERR_ARG), (dict(saved=0x90000000), ar.AR_ERR_ARG),
    (dict(ld_dx=63), ar.AR_ERR_ARG), (dict(dh=A + 1), ar.AR_ERR_ARG)])
def test_ffn_backward_refusals(kw, code):
    assert ffn_bwd(**kw) == code


def test_ffn_without_tokens_is_done():
    assert ffn(tokens=0, x=None, h=None) == ar.AR_OK
    assert ffn_bwd(tokens=0, dx=None, dwg=None, dwu=None, ws=None) == ar.AR_OK


def test_ffn_tensor_checks():
    t = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        ar.gated_ffn(t, t, t)
    with pytest.raises(ValueError, match="GPU"):
        ar.gated_ffn_backward(t, t, t, t, t)


@pytest.mark.parametrize("act", ("silu", "gelu", "relu"))
def test_ffn_plain_gradient_is_the_difference(act):
    torch.manual_seed(1)
    rnd = lambda *s: torch.randn(*s, dtype=torch.float64)  # noqa: E731
    v, dh, h = dict(x=rnd(5, 8), wg=rnd(6, 8), wu=rnd(6, 8)), rnd(5, 6), 1e-6
    loss = lambda u: float((dh * oo.gated_ffn(u["x"], u["wg"], u["wu"], act)[0]).sum())  # noqa: E731
    grads = oo.gated_ffn_backward(dh, v["x"], v["wg"], v["wu"], act)
    for name, g in zip(("x", "wg", "wu"), grads):
        e = rnd(*v[name].shape)
        fd = (loss({**v, name: v[name] + h * e}) - loss({**v, name: v[name] - h * e})) / (2 * h)
        assert abs(fd - float((g * e).sum())) < 1e-6 * (1 + abs(fd)), name


def ortho(i=A, o=B, ws=0x90000000, nbytes=None, coefs=(3.4, -4.8, 2.0), **kw):
    f = dict(batch=2, rows=8, cols=16, dtype=0, steps=1, eps=1e-7, scale=1.0)
    f.update(kw)
    d = ops.ar_ortho_desc(**f)
    if coefs is not None:
        d.coefs = (ctypes.c_float * (3 * 16))(*(tuple(coefs) * 16))
    L = ops._lib()
    n = L.ar_orthogonalize_workspace(ctypes.byref(d)) if nbytes is None else nbytes
    return L.ar_orthogonalize(ctypes.byref(d), i, o, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), ar.AR_ERR_UNSUPPORTED), (dict(rows=0), ar.AR_ERR_ARG), (dict(cols=65537), ar.AR_ERR_ARG),
    (dict(steps=0), ar.AR_ERR_ARG), (dict(steps=17), ar.AR_ERR_ARG), (dict(coefs=None), ar.AR_ERR_ARG),
    (dict(coefs=(float("nan"), 0, 0)), ar.AR_ERR_ARG), (dict(coefs=(5000.0, 0, 0)), ar.AR_ERR_ARG),
    (dict(coefs=(20.0, 0, 0), steps=3), ar.AR_ERR_ARG), (dict(eps=-1.0), ar.AR_ERR_ARG), (dict(scale=float("inf")), ar.AR_ERR_ARG),
    (dict(ld_in=15), ar.AR_ERR_ARG), (dict(stride_in=100), ar.AR_ERR_ARG), (dict(stride_out=16, ld_out=20), ar.AR_ERR_ARG),
    (dict(i=None), ar.AR_ERR_ARG), (dict(o=B + 2), ar.AR_ERR_ARG), (dict(o=A + 64), ar.AR_ERR_ARG), (dict(o=A, ld_out=20), ar.AR_ERR_ARG),
    (dict(ws=None), ar.AR_ERR_SCRATCH), (dict(nbytes=64), ar.AR_ERR_SCRATCH), (dict(ws=0x90000020), ar.AR_ERR_ARG),
    (dict(ws=A), ar.AR_ERR_ARG)])
def test_ortho_refusals(kw, code):
    assert ortho(**kw) == code
    assert ar.ar_last_error() == code


def test_ortho_without_matrices_is_done():
    assert ortho(batch=0, i=None, o=None, ws=None) == ar.AR_OK


def test_ortho_tensor_checks():
    with pytest.raises(ValueError, match="GPU"):
        ar.orthogonalize(torch.zeros(4, 8))


def test_ffn_in_runs_needs_its_workspace():
    """One tile and a long dim: the sums are taken in runs, which lie in the
    workspace; a large hidden takes them in one piece."""
    L = ops._lib()
    d = ops.ar_ffn_desc(tokens=4, dim=4096, hidden=64, dtype=1, act=0)
    copies = 2 * 4096 * (4 + 2 * 64)
    assert L.ar_gated_ffn_workspace(ctypes.byref(d)) > copies
    assert (L.ar_gated_ffn_workspace(ctypes.byref(d)) - copies) % (2 * 4 * 64 * 4) == 0
    big = dict(x=0x100000000, wg=0x200000000, wu=0x300000000, h=0x400000000, dim=4096, hidden=64)
    assert ffn(**big) == ar.AR_ERR_SCRATCH
    assert ffn(ws=0x500000000, nbytes=1024, **big) == ar.AR_ERR_SCRATCH
    assert ffn(ws=0x500000008, nbytes=1 << 30, **big) == ar.AR_ERR_ARG
    assert ffn(ws=0x400000000, nbytes=1 << 30, **big) == ar.AR_ERR_ARG
    d = ops.ar_ffn_desc(tokens=4, dim=4096, hidden=16384, dtype=1, act=0)
    assert L.ar_gated_ffn_workspace(ctypes.byref(d)) == 2 * 4096 * (4 + 2 * 16384)
