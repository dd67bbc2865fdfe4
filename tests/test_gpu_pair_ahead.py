"""The gated feed-forward block's 256 x 256 tiles with two buffers and with three, against 64
bits and each other, with the tolerances of test_gpu_ffn.py.  tests/test_pair_ahead.py
holds the sizes to the tiles."""
from __future__ import annotations

import pytest

from gemm_shapes_ahead import BOTH
from gpu_helpers import say
from test_gpu_ffn import check, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,t,d,f", BOTH)
def test_both(act, t, d, f):
    """`check` has h with the projections saved and without, bit for bit."""
    say(f"ffn {t} x {d} x {f} {act}")
    check(*inputs(t, d, f, seed=6), act)
