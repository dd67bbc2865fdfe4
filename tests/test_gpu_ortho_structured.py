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


def signs(m, n, rank, seed=4):
    g = torch.Generator().manual_seed(seed)
    return torch.sign(torch.randn(m, rank, generator=g)) @ torch.sign(torch.randn(rank, n, generator=g))


def low_rank(m, n, rank, seed=5):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(m, rank, generator=g) @ torch.randn(rank, n, generator=g)


def hadamard(m, n):
    h = torch.ones(1, 1)
    while len(h) < n:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)])
    return h[:m]


STRUCTURED = {
    "constant 700 x 700": lambda: torch.ones(700, 700),
    "constant 572 x 2158": lambda: 0.3 * torch.ones(572, 2158),
    "constant 1672 x 1062": lambda: 1e-4 * torch.ones(1672, 1062),
    "hadamard 512 x 1024": lambda: hadamard(512, 1024),
    "signs of rank 1": lambda: signs(400, 400, 1),
    "signs of rank 2": lambda: signs(500, 500, 2),
    "signs of rank 3": lambda: signs(400, 400, 3),
    "signs of rank 3, tall": lambda: signs(900, 400, 3),
    "blocks of 4 ones": lambda: torch.block_diag(*[torch.ones(4, 4)] * 100),
    "blocks of 16 ones": lambda: torch.block_diag(*[torch.ones(16, 16)] * 30),
    "two diagonals": lambda: torch.eye(400) + 0.5 * torch.diag(torch.ones(399), 1),
    "columns' own scales": lambda: torch.ones(400, 600) * torch.linspace(0.5, 3, 600),
    "repeated columns": lambda: low_rank(300, 3, 3).repeat_interleave(200, 1),
    "rank 16": lambda: low_rank(300, 300, 16),
    "rank 60": lambda: low_rank(300, 500, 60),
    "rows of zeros": lambda: low_rank(900, 900, 900) * (torch.arange(900) % 3 == 0)[:, None],
    "a step's triangle": lambda: torch.ones(400, 400).triu(),
}


@pytest.mark.parametrize("kind", list(STRUCTURED))
def test_few_magnitudes_and_low_rank(kind):
    """With every rounding of the one plane, and no other error, modelled in 64 bits,
    results of 50 kinds, these among them, were off by at most 2.8e-3 of their norm (blocks of
    ones; with nearest rounding and diagonals from the rounded plane 9.5e-3, a
    constant).  3e-3 is asked beside the result's own rounding to bf16."""
    say(f"ortho {kind}")
    off, rounding = off_by(STRUCTURED[kind]())
    assert off <= rounding + 3e-3, (off, rounding)
