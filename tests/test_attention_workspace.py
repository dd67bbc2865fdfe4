"""The workspace that attention's backward pass is told to have is enough for the calls
that it is meant for (no GPU)."""
from __future__ import annotations

import ctypes
import itertools

import pytest

import paper_2603_11438_amd as ar
from paper_2603_11438_amd import ops
from test_ops_host import built_lib  # noqa: F401

SIZES = list(itertools.product((1, 33, 90, 128, 300, 512, 777, 2048, 4096), (1, 90, 300, 777, 2048, 9000, 33000),
                               ((1, 1), (8, 1), (8, 8), (32, 8), (6, 2)), (64, 80, 128), (1, 2, 7)))


def wanted(queries, keys, heads, kv_heads, dim, sequences, causal):
    """What a call of packed_attention_backward asks of its workspace."""
    d = ops.ar_attention_desc(sequences=sequences, tokens_q=queries, tokens_k=keys, heads=heads, kv_heads=kv_heads, dim=dim,
                              dtype=ar.AR_BFLOAT16, flags=ops.AR_ATTN_CAUSAL if causal else 0, scale=dim ** -0.5)
    return ops._lib().ar_attention_backward_workspace(ctypes.byref(d))


@pytest.mark.parametrize("causal", (True, False))
def test_enough_for_causal_calls_and_others(causal):
    for q, k, (h, hk), dim, sequences in SIZES:
        need = wanted(q, k, h, hk, dim, sequences, causal)
        named = ar.packed_attention_backward_workspace(q, k, h, hk, dim, sequences)
        assert named >= need > 0, (q, k, h, hk, dim, sequences)
        assert ar.packed_attention_backward_workspace(q, k, h, hk, dim, sequences, causal=causal) == need


def test_where_causal_calls_need_more():
    """One sequence, 777 tokens of 32 heads over 8: its gradients are summed up in more runs."""
    assert wanted(777, 777, 32, 8, 128, 1, True) > wanted(777, 777, 32, 8, 128, 1, False)
    assert ar.packed_attention_backward_workspace(777, 777, 32, 8, 128) == wanted(777, 777, 32, 8, 128, 1, True)
