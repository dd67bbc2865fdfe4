"""Orthogonalised updates of bf16 matrices whose elements share few magnitudes,
so that a plane's rounding errors need not average, against the definition in 64
bits (oracle/ops_oracle.py).  All have a short side above 256: the products take
one plane there."""
from __future__ import annotations

import pytest
import torch

import paper_2603_11438_amd as ar
from gpu_helpers import say
from oracle import ops_oracle as oo

pytestmark = pytest.mark.gpu

COEFS = ((3.4445, -4.7750, 2.0315),) * 5


def off_by(x):
    """The result's error and that of rounding the exact one to bf16, of the exact norm."""
    x = x.contiguous().bfloat16().cuda()
    want = oo.orthogonalize(x, COEFS)
    got = ar.orthogonalize(x).cpu().double()
    assert bool(torch.isfinite(got).all())
    return float((got - want).norm() / want.norm()), float((want.bfloat16().double() - want).norm() / want.norm())


def one_a_row(m, n, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.zeros(m, n)
    x[torch.arange(m), torch.randperm(n, generator=g)[:m]] = 1.0 - 2.0 * torch.randint(0, 2, (m,), generator=g)
    return x


@pytest.mark.parametrize("m,n,scale", [(360, 360, 1.0), (482, 482, 1e-3), (300, 1000, 7.0), (1410, 700, 0.3), (2100, 2100, 1.0)])
def test_one_element_a_row(m, n, scale):
    """A and B are diagonal matrices, which stay in fp32: beside the result's own
    rounding there are only fp32's, which five steps amplify to far below 1e-4."""
    for x in (torch.eye(m, n), one_a_row(m, n, m) if m <= n else one_a_row(n, m, m).t()):
        say(f"ortho one element a row {m} x {n}")
        off, rounding = off_by(scale * x)
        assert off <= 1.02 * rounding + 1e-4, (off, rounding)
