"""Attention's requests that are refused before anything is launched, and its plain
form's gradients against differences (no GPU)."""
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
Q, K, V, O, DO, LSE, SQ, SK, DQ, DK, DV, WS = (0x10000000 * k for k in range(1, 13))


def desc(**kw):
    f = dict(sequences=2, tokens_q=64, tokens_k=64, heads=4, kv_heads=2, dim=64, dtype=1, flags=1, scale=0.125)
    return ops.ar_attention_desc(**{**f, **kw})


def forward(q=Q, k=K, v=V, sq=SQ, sk=SK, o=O, lse=None, ws=WS, nbytes=1 << 30, **kw):
    return ops._lib().ar_attention(ctypes.byref(desc(**kw)), q, k, v, sq, sk, o, lse, ws, nbytes, None)


BAD_DESC = [
    (dict(dtype=0), ar.AR_ERR_UNSUPPORTED), (dict(dim=129), ar.AR_ERR_UNSUPPORTED), (dict(dim=0), ar.AR_ERR_ARG), (dict(heads=0), ar.AR_ERR_ARG),
    (dict(kv_heads=0), ar.AR_ERR_ARG), (dict(kv_heads=3), ar.AR_ERR_ARG), (dict(kv_heads=8), ar.AR_ERR_ARG), (dict(flags=4), ar.AR_ERR_ARG),
    (dict(scale=0.0), ar.AR_ERR_ARG), (dict(scale=-1.0), ar.AR_ERR_ARG), (dict(scale=float("nan")), ar.AR_ERR_ARG),
    (dict(scale=float("inf")), ar.AR_ERR_ARG), (dict(scale=1e-38), ar.AR_ERR_ARG), (dict(scale=1e38), ar.AR_ERR_ARG), (dict(tokens_q=1 << 30), ar.AR_ERR_ARG), (dict(tokens_k=1 << 31), ar.AR_ERR_ARG),
    (dict(sequences=(1 << 20) + 1), ar.AR_ERR_ARG), (dict(tokens_q=(1 << 28) + 1), ar.AR_ERR_ARG), (dict(heads=1 << 17), ar.AR_ERR_ARG), (dict(sq=None), ar.AR_ERR_ARG), (dict(sk=None), ar.AR_ERR_ARG),
    (dict(sq=None, sk=None), ar.AR_ERR_ARG), (dict(sq=SQ + 2), ar.AR_ERR_ARG), (dict(q=None), ar.AR_ERR_ARG), (dict(q=Q + 1), ar.AR_ERR_ARG),
    (dict(v=None), ar.AR_ERR_ARG), (dict(hs_q=63), ar.AR_ERR_ARG), (dict(ld_k=63), ar.AR_ERR_ARG), (dict(ld_k=100), ar.AR_ERR_ARG),
    (dict(ld_v=1 << 50), ar.AR_ERR_ARG), (dict(o=None), ar.AR_ERR_ARG)]


@pytest.mark.parametrize("kw,code", BAD_DESC + [
    (dict(o=Q), ar.AR_ERR_ARG), (dict(o=K + 128), ar.AR_ERR_ARG), (dict(o=SQ), ar.AR_ERR_ARG), (dict(lse=O), ar.AR_ERR_ARG),
    (dict(lse=V), ar.AR_ERR_ARG), (dict(lse=LSE + 2), ar.AR_ERR_ARG), (dict(q=Q + 2, ws=None), ar.AR_ERR_SCRATCH),
    (dict(dim=60, nbytes=64), ar.AR_ERR_SCRATCH), (dict(q=Q + 2, ws=WS + 16), ar.AR_ERR_ARG), (dict(q=Q + 2, ws=K), ar.AR_ERR_ARG),
    (dict(q=Q + 2, ws=O), ar.AR_ERR_ARG)])
def test_forward_refusals(kw, code):
    assert forward(**kw) == code
    assert ar.ar_last_error() == code


def backward(do=DO, q=Q, k=K, v=V, o=O, lse=LSE, sq=SQ, sk=SK, dq=DQ, dk=DK, dv=DV, ws=WS, nbytes=1 << 30, **kw):
    return ops._lib().ar_attention_backward(ctypes.byref(desc(**kw)), do, q, k, v, o, lse, sq, sk, dq, dk, dv, ws, nbytes, None)


@pytest.mark.parametrize("kw,code", BAD_DESC + [
    (dict(do=None), ar.AR_ERR_ARG), (dict(lse=None), ar.AR_ERR_ARG), (dict(dk=None), ar.AR_ERR_ARG), (dict(dv=None), ar.AR_ERR_ARG),
    (dict(dq=Q), ar.AR_ERR_ARG), (dict(dk=DV), ar.AR_ERR_ARG), (dict(dv=DO), ar.AR_ERR_ARG), (dict(dq=LSE), ar.AR_ERR_ARG),
    (dict(hs_dq=8), ar.AR_ERR_ARG), (dict(ld_dk=70), ar.AR_ERR_ARG), (dict(ws=None), ar.AR_ERR_SCRATCH), (dict(nbytes=100), ar.AR_ERR_SCRATCH),
    (dict(ws=WS + 128), ar.AR_ERR_ARG), (dict(ws=LSE), ar.AR_ERR_ARG), (dict(ws=DK), ar.AR_ERR_ARG)])
def test_backward_refusals(kw, code):
    assert backward(**kw) == code


def test_nothing_to_do():
    assert forward(sequences=0, q=None, o=None) == ar.AR_OK
    assert forward(tokens_q=0, q=None, o=None) == ar.AR_OK
    assert backward(sequences=0, q=None, ws=None) == ar.AR_OK
    assert backward(dq=None, dk=None, dv=None, ws=None) == ar.AR_OK


def test_tensor_checks():
    t = torch.zeros(4, 2, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        ar.packed_attention(t, t, t)
    with pytest.raises(ValueError, match="GPU"):
        ar.packed_attention_backward(t, t, t, t, t, t)


@pytest.mark.parametrize("causal", (True, False))
def test_plain_gradient_is_the_difference(causal):
    torch.manual_seed(2)
    rnd = lambda *s: torch.randn(*s, dtype=torch.float64)  # noqa: E731
    sq, sk, step = [0, 5, 5, 9], [0, 4, 6, 13], 1e-6
    x = {"q": rnd(9, 4, 6), "k": rnd(13, 2, 6), "v": rnd(13, 2, 6)}
    do = rnd(9, 4, 6)
    loss = lambda u: float((do * oo.attention(u["q"], u["k"], u["v"], sq, sk, causal)["o"][0]).sum())  # noqa: E731
    grads = oo.attention(x["q"], x["k"], x["v"], sq, sk, causal, do=do)
    for name in x:
        e = rnd(*x[name].shape)
        fd = (loss({**x, name: x[name] + step * e}) - loss({**x, name: x[name] - step * e})) / (2 * step)
        assert abs(fd - float((grads["d" + name][0] * e).sum())) < 1e-6 * (1 + abs(fd)), name
