"""Which places of its tensors attention takes (no GPU).  The addresses are never followed:
without a workspace a call that would be taken is AR_ERR_SCRATCH, one whose results overlap
anything AR_ERR_ARG before that."""
from __future__ import annotations

import ctypes

import pytest

import paper_2603_11438_amd as ar
from paper_2603_11438_amd import ops
from test_ops_host import built_lib  # noqa: F401

A, FAR = 0x10000000, 0x1000000  # no tensor here is so long
TOKENS, HEADS, DIM = 5, 3, 12  # no multiple of eight: inputs are copied, so the forward pass wants a workspace too
NAMES = ("q", "k", "v", "o", "dout", "dq", "dk", "dv")


def answer(fused, tokens=TOKENS, kv_heads=HEADS, backward=True):
    """fused: {name: (elements behind the common begin, ld, hs)}; the other tensors lie far apart."""
    heads = {n: kv_heads if n in ("k", "v", "dk", "dv") else HEADS for n in NAMES}
    d = ops.ar_attention_desc(sequences=1, tokens_q=tokens, tokens_k=tokens, heads=HEADS, kv_heads=kv_heads, dim=DIM, dtype=1, flags=1, scale=1.0)
    at = {n: A + FAR * (k + 1) for k, n in enumerate(NAMES)}
    for n, (first, ld, hs) in fused.items():
        at[n] = A + 2 * first
        setattr(d, "ld_" + n, ld), setattr(d, "hs_" + n, hs)
    L, lse = ops._lib(), A + 100 * FAR
    if backward:
        rc = L.ar_attention_backward(ctypes.byref(d), at["dout"], at["q"], at["k"], at["v"], at["o"], lse, None, None, at["dq"], at["dk"],
                                     at["dv"], None, 0, None)
    else:
        rc = L.ar_attention(ctypes.byref(d), at["q"], at["k"], at["v"], None, None, at["o"], lse, None, 0, None)
    assert rc in (ar.AR_ERR_SCRATCH, ar.AR_ERR_ARG)
    elements = {n: {first + t * ld + h * hs + e for t in range(tokens) for h in range(heads[n]) for e in range(DIM)}
                for n, (first, ld, hs) in fused.items()}
    results = ("dq", "dk", "dv") if backward else ("o",)
    shared = any(elements[a] & elements[b] for a in fused if a in results for b in fused if a != b)
    return rc == ar.AR_ERR_SCRATCH, not shared


D = DIM
# (tokens, heads, 3, dim), (tokens, 3, heads, dim), (heads, tokens, 3, dim), and with room beside
TRIPLES = [
    [(0, 9 * D, 3 * D), (D, 9 * D, 3 * D), (2 * D, 9 * D, 3 * D)],
    [(2 * D, 9 * D, 3 * D), (0, 9 * D, 3 * D), (D, 9 * D, 3 * D)],
    [(0, 9 * D, D), (3 * D, 9 * D, D), (6 * D, 9 * D, D)],
    [(0, 3 * D, 3 * D * TOKENS), (D, 3 * D, 3 * D * TOKENS), (2 * D, 3 * D, 3 * D * TOKENS)],
    [(0, 9 * D + 7, 3 * D), (D, 9 * D + 7, 3 * D), (2 * D, 9 * D + 7, 3 * D)],
    [(0, 12 * D, 4 * D), (D + 3, 12 * D, 4 * D), (3 * D - 1, 12 * D, 4 * D)],
]


@pytest.mark.parametrize("places", TRIPLES, ids=str)
@pytest.mark.parametrize("tokens", [1, TOKENS])
def test_parts_of_one_tensor_are_taken(places, tokens):
    assert answer(dict(zip(("dq", "dk", "dv"), places)), tokens) == (True, True)
    assert answer(dict(zip(("q", "dq", "dout"), places)), tokens) == (True, True)
    assert answer(dict(zip(("q", "k", "o"), places)), tokens, backward=False) == (True, True)


@pytest.mark.parametrize("by", [-1, 1, -D, D, 3 * D, 9 * D, -9 * D, 10 * D, 18 * D])
@pytest.mark.parametrize("places", TRIPLES, ids=str)
def test_shifted(places, by):
    """As the elements say, or refused."""
    second = (places[1][0] + by, *places[1][1:])
    for names, backward in ((("dq", "dk"), True), (("dk", "v"), True), (("q", "o"), False)):
        taken, apart = answer(dict(zip(names, (places[0], second))), backward=backward)
        assert taken == apart


def test_key_heads_that_are_fewer():
    """k and v, and their gradients, with one head in three, beside each other and in turn."""
    assert answer({"dk": (0, 2 * D, 0), "dv": (D, 2 * D, 0)}, kv_heads=1) == (True, True)
    assert answer({"dk": (0, 2 * D, 0), "dv": (D - 1, 2 * D, 0)}, kv_heads=1) == (False, False)
    assert answer({"dq": (0, 5 * D, D), "dk": (3 * D, 5 * D, 0), "dv": (4 * D, 5 * D, 0)}, kv_heads=1) == (True, True)


def test_other_strides_are_refused_where_addresses_cross():
    assert answer({"dk": (0, 9 * D, 3 * D), "dv": (D, 9 * D, 4 * D)})[0] is False
    assert answer({"dk": (0, 9 * D, 3 * D), "dv": (D, 10 * D, 3 * D)})[0] is False
    assert answer({"dk": (0, 9 * D, 3 * D), "dv": (45 * D, 10 * D, 3 * D)}) == (True, True)
