"""Sizes of the workspaces that calls with given operands use (no GPU)."""
from __future__ import annotations

import ctypes

import pytest

from paper_2603_11438_amd import ops
from test_ops_host import built_lib  # noqa: F401

A = 0x100000000


def need(x=A, wg=2 * A, wu=3 * A, **kw):
    d = ops.ar_ffn_desc(**{**dict(tokens=100, dim=64, hidden=320, dtype=1, act=0), **kw})
    L = ops._lib()
    got = L.ar_gated_ffn_workspace_for(ctypes.byref(d), x, wg, wu)
    assert got <= L.ar_gated_ffn_workspace(ctypes.byref(d))
    return got


@pytest.mark.parametrize("kw,rows,cols", [
    (dict(), 0, 0), (dict(x=A + 2), 100, 64), (dict(wg=2 * A + 8), 320, 64), (dict(x=A + 2, wu=3 * A + 4), 420, 64), (dict(ld_x=70), 100, 64),
    (dict(ld_x=72), 0, 0), (dict(ld_w_up=65), 320, 64), (dict(dim=60), 740, 64), (dict(dim=72, ld_x=73), 100, 128)])
def test_copies_that_the_operands_ask_for(kw, rows, cols):
    assert need(**kw) == rows * cols * 2


def test_runs():
    assert need(tokens=4, dim=4096, hidden=64) % (2 * 4 * 64 * 4) == 0
    assert 0 < need(tokens=4, dim=4096, hidden=64) <= 32 * 2 * 4 * 64 * 4
    assert need(tokens=4, dim=4096, hidden=64, x=A + 2) == need(tokens=4, dim=4096, hidden=64) + 4 * 4096 * 2


def test_nothing_where_the_call_is_refused_or_empty():
    assert need(tokens=0) == 0 and need(dtype=0) == 0 and need(act=9) == 0 and need(dim=0) == 0
