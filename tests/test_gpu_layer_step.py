"""The operators and the collective together, as a shared block's training step
uses them, against the block in one piece in fp64 on the CPU.

Tolerance, of each result's norm: every tensor that is kept in bf16 on the way
(h, the partial and joined sums, s and out; dout, dy, dh, the products' dG and
dU, the partial and joined dx) is off by at most 2^-8 / sqrt(3) = 2.3e-3 of its
norm, a dozen of them in a chain by 8e-3; 2e-2 leaves room for where the norms'
backward passes cancel."""
from __future__ import annotations

import pytest
import torch

from gpu_helpers import say

pytestmark = pytest.mark.gpu

TOL = 2e-2


def plain(block, x, residual, target, alpha):
    """Loss and gradients in fp64, from the same weights and inputs."""
    wide = lambda t: t.detach().cpu().double().requires_grad_()  # noqa: E731
    x, residual = wide(x), wide(residual)
    wg, wu = wide(torch.cat(block.wg)), wide(torch.cat(block.wu))
    wd, post, pre = wide(torch.cat(block.wd, 1)), wide(block.post), wide(block.pre)
    norm = lambda v, w: v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6) * w  # noqa: E731
    g = x @ wg.t()
    y = (g * torch.sigmoid(g) * (x @ wu.t())) @ wd.t()
    s = alpha * residual + norm(y, post)
    out = norm(s, pre)
    loss = (out - target.cpu().double()).square().mean()
    loss.backward()
    return {"loss": loss.detach(), "y": y.detach(), "s": s.detach(), "out": out.detach(), "dx": x.grad, "dresidual": residual.grad,
            "dpost": post.grad, "dpre": pre.grad, "dwg": wg.grad, "dwu": wu.grad, "dwd": wd.grad}


@pytest.mark.parametrize("ranks,tokens,dim,hidden", [(4, 96, 256, 512), (2, 130, 200, 328), (1, 33, 72, 64), (8, 1, 128, 256)])
def test_block(ranks, tokens, dim, hidden):
    from paper_2603_11438_amd.layer_step import Block

    say("block", ranks, tokens, dim, hidden)
    block = Block(ranks, dim, hidden, seed=ranks)
    gen = torch.Generator().manual_seed(7)
    x, residual, target = (torch.randn(tokens, dim, generator=gen).cuda() for _ in range(3))
    x, residual = x.bfloat16(), residual.bfloat16()
    got = block.gradients(x, residual, target, alpha=0.5)
    want = plain(block, x, residual, target, 0.5)
    assert all(torch.equal(t, got["y"][0]) for t in got["y"]), "the ranks' joined sums differ"
    got |= {"y": got["y"][0], "dwg": torch.cat(got["dwg"]), "dwu": torch.cat(got["dwu"]), "dwd": torch.cat(got["dwd"], 1)}
    for name, w in want.items():
        off = float((got[name].cpu().double() - w).norm() / w.norm())
        assert off <= TOL, f"{name} off by {off:.3g}"


def test_losses_fall():
    from paper_2603_11438_amd import layer_step

    losses = layer_step.run(ranks=4, tokens=256, dim=256, hidden=512, steps=4, say=say)
    assert all(b < a for a, b in zip(losses, losses[1:])), losses


def test_uneven_split_is_refused():
    from paper_2603_11438_amd.layer_step import Block

    with pytest.raises(ValueError):
        Block(3, 64, 100)
