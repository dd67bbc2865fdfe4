"""Which places of input and output orthogonalize takes (no GPU).  The addresses are
never followed: without a workspace a call that would be taken is AR_ERR_SCRATCH, one
whose places overlap AR_ERR_ARG before that."""
from __future__ import annotations

import pytest

import paper_2603_11438_amd as ar
from test_ops_host import built_lib, ortho  # noqa: F401

A = 0x10000000
ROWS, COLS = 8, 16  # fp32


def taken(batch, at, ld, stride, at_out, ld_out=None, stride_out=None):
    """at_out: elements behind the input's begin at which the output begins."""
    rc = ortho(i=A + 4 * at, o=A + 4 * at_out, ws=None, batch=batch, rows=ROWS, cols=COLS, ld_in=ld, stride_in=stride,
               ld_out=ld if ld_out is None else ld_out, stride_out=stride if stride_out is None else stride_out)
    assert rc in (ar.AR_ERR_SCRATCH, ar.AR_ERR_ARG)
    return rc == ar.AR_ERR_SCRATCH


def shares(batch, at, ld, stride, at_out, ld_out=None, stride_out=None):
    """By enumeration."""
    def elements(first, ld, stride):
        return {first + b * stride + r * ld + c for b in range(batch) for r in range(ROWS) for c in range(COLS)}

    return bool(elements(at, ld, stride) & elements(at_out, ld if ld_out is None else ld_out, stride if stride_out is None else stride_out))


PLACES = [
    # batch, at, ld, stride, at_out[, ld_out, stride_out]
    (1, 0, 40, 0, 16), (1, 0, 40, 0, 24), (1, 24, 40, 0, 0), (1, 0, 40, 0, 15), (1, 0, 40, 0, 25), (1, 0, 32, 0, 16),
    (3, 0, 40, 320, 16), (3, 0, 40, 320, 20), (3, 0, 40, 400, 20), (3, 0, 40, 320, 8),  # one after another, beside each other
    (3, 0, 128, 32, 16), (3, 16, 128, 32, 0), (3, 0, 128, 32, 15), (3, 0, 200, 16, 48), (3, 0, 200, 16, 32),  # side by side
    (3, 0, 16, 128, 128), (3, 0, 16, 128, 384), (3, 0, 16, 256, 128), (3, 0, 16, 256, 100),  # in turn
    (3, 0, 40, 320, 16, 40, 400), (3, 0, 200, 16, 48, 200, 24), (3, 0, 200, 32, 16, 200, 48), (2, 0, 128, 32, 16, 128, 80),
]


@pytest.mark.parametrize("place", PLACES)
def test_places(place):
    assert taken(*place) == (not shares(*place))


def test_in_place():
    assert taken(3, 0, 40, 320, 0) and taken(3, 0, 200, 16, 0) and taken(1, 0, 40, 320, 0, 40, 999)
    assert not taken(3, 0, 40, 320, 0, 40, 400) and not taken(1, 0, 40, 0, 0, 41, 0)


def test_many_matrices():
    assert taken(60000, 0, 40, 320, 20) and not taken(60000, 0, 40, 320, 8)
    assert taken(2000, 0, 40, 320, 20, 40, 400) == (not shares(40, 0, 40, 320, 20, 40, 400))
