"""The gated feed-forward block where projections leave fp32's range."""
from __future__ import annotations

import pytest
import torch

import paper_2603_11438_amd as ar
from gpu_helpers import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,dim", [(3, 64), (70, 64), (8, 2048)])
def test_relu_of_minus_infinity_is_zero(tokens, dim):
    """max(g, 0) is 0 at -inf and inf at inf, and its gradient 0 and 1: the token's own
    projections overflow, everything it meets is finite.  In one piece and in runs."""
    say(f"relu of infinities {tokens} x {dim}")
    hidden = 24
    x = torch.full((tokens, dim), 2.0 ** 120).bfloat16().cuda()
    wg = torch.full((hidden, dim), -(2.0 ** 10)).bfloat16().cuda()
    wg[::2] = 0.0
    wg[5] = 2.0 ** 10
    wu = torch.full((hidden, dim), 2.0 ** -120).bfloat16().cuda()
    h, saved = ar.gated_ffn(x, wg, wu, act="relu", save=True)
    want = torch.zeros(hidden)
    want[5] = float("inf")
    assert torch.equal(saved[0].cpu().amin(0), torch.tensor([0.0 if k % 2 == 0 else float("inf") if k == 5 else -float("inf") for k in range(hidden)]))
    assert torch.equal(h.float().cpu(), want.expand(tokens, hidden))
    dh = torch.ones_like(h)
    dh[:, 5] = 0
    finite = [k for k in range(hidden) if k != 5]  # that column's dU is 0 times inf
    dx, dwg, dwu = ar.gated_ffn_backward(dh[:, finite].contiguous(), x, wg[finite], wu[finite], saved[:, :, finite].contiguous(), act="relu")
    assert bool((dx == 0).all()) and bool((dwg == 0).all()) and bool((dwu == 0).all())


def test_relu_keeps_nan():
    x = torch.ones(4, 64).bfloat16().cuda()
    x[2, 7] = float("nan")
    w = torch.ones(8, 64).bfloat16().cuda()
    h = ar.gated_ffn(x, -w, w, act="relu").float()
    assert bool(torch.isnan(h[2]).all()) and bool((h[[0, 1, 3]] == 0).all())
