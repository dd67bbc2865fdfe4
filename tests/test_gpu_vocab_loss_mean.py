"""Gradients of a masked mean: dloss the same for each token that counts, and 0 or anything
for those that have no class, the first ones among them."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2603_11438_amd as ar
from gpu_helpers import say
from oracle import ops_oracle as oo

pytestmark = pytest.mark.gpu

COUNT = 255  # 1 / 255 = 1.00392 / 256 lies half-way between two bf16 values


def inputs(tokens, dim, classes, ignored, seed=0):
    """`ignored` tokens in front, and some of the rest, without a class: COUNT have one."""
    g = torch.Generator().manual_seed(seed)
    x, w = torch.randn(tokens, dim, generator=g).bfloat16(), (0.1 / math.sqrt(dim) * torch.randn(classes, dim, generator=g)).bfloat16()
    target = torch.full((tokens,), -100)
    counting = ignored + torch.cat([torch.zeros(1, dtype=torch.int64), 1 + torch.randperm(tokens - ignored - 1, generator=g)[:COUNT - 1]])
    target[counting] = torch.randint(0, classes, (COUNT,), generator=g)
    return x.cuda(), w.cuda(), target.cuda(), torch.where(target >= 0, 1.0 / COUNT, 0.0).cuda()


def gradients(x, w, target, dloss, **kw):
    return ar.vocab_loss_backward(dloss, x, w, target, ar.vocab_loss(x, w, target)[1], **kw)


# tokens, dim, classes, tokens without a class in front: with a few tokens, with many, in one look and in several
SIZES = [(255, 64, 5001, 0), (256, 64, 5001, 1), (300, 72, 5001, 40), (700, 64, 3001, 445), (1024, 64, 5001, 700), (1025, 64, 5001, 1),
         (1100, 64, 3001, 800), (5000, 64, 3001, 4300), (13000, 64, 1001, 12500), (300, 1, 70000, 30), (1000, 16, 280001, 500)]


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_errors_are_not_all_in_one_direction(size):
    """In norm.  A value rounded to bf16 is off by at most 2^-8 of itself, evenly spread, so
    by 2^-8 / sqrt(3) = 2.26e-3 in the mean square at most: that is the result's rounding.
    An operand dz is (p - 1) 2^-8 at a target, which rounds to -2^-8 (1 - p) within p / 2 or
    half a step: with logits of 0.1, p is below 2 / classes, so within 2.1e-3 at 1001
    classes and 7e-4 from 3001 on, and p 2^-8 elsewhere, all of them together
    sqrt(classes) p of the targets' weight, at most 0.07, times 2.26e-3.  Together below
    3e-3 (1001: 3.4e-3).  Rounded without a factor taken out, 1 / 255 is off by 3.9e-3 at
    every target, which with the result's rounding is 4.2e-3 and more."""
    say("mean", size)
    x, w, target, dloss = inputs(*size)
    want = oo.vocab_loss(x, w, target, dloss, "cuda" if size[0] * size[2] > 1 << 21 else "cpu")
    for name, got in zip(("dx", "dw"), gradients(x, w, target, dloss)):
        value, bound = (t.to(got.device) for t in want[name])
        off = got.double() - value
        assert bool((off.abs() <= bound).all()), name
        relative = float(off.norm() / value.norm())
        say(name, relative)
        assert relative < (3.4e-3 if size[2] < 3000 else 3e-3), name


@pytest.mark.parametrize("size", [(300, 64, 1001, 40), (1300, 64, 1001, 1000), (9000, 16, 501, 8500)], ids=str)
def test_dloss_of_tokens_without_a_class_does_not_count(size):
    say("whatever", size)
    x, w, target, dloss = inputs(*size)
    want = gradients(x, w, target, dloss)
    for value in (0.0, -0.7, 1e-40, math.inf, math.nan, 3e38):
        dloss[target < 0] = value
        for a, b in zip(gradients(x, w, target, dloss), want):
            assert torch.equal(a, b), value


@pytest.mark.parametrize("size", [(300, 64, 1001, 0), (1300, 64, 1001, 0)], ids=str)
def test_what_leads(size):
    """A dloss of 0 does not, of either sign; powers of two in all of them change no bits of
    the results but their exponents; tokens' dloss at a stride; a rank's rows."""
    say("leads", size)
    x, w, target, dloss = inputs(*size)
    dloss[:7] = 0.0
    dloss[3] = -0.0
    want = gradients(x, w, target, dloss)
    for a, b in zip(gradients(x, w, target, dloss * 2.0 ** 20), want):
        assert torch.equal(a.float(), b.float() * 2.0 ** 20)
    for a, b in zip(gradients(x, w, target, -dloss), want):
        assert torch.equal(a, -b)
    apart = torch.full((size[0], 3), math.nan, device="cuda")
    apart[:, 1] = dloss
    for a, b in zip(gradients(x, w, target, apart[:, 1]), want):
        assert torch.equal(a, b)
    lse = ar.vocab_loss(x, w, target)[1]
    # a rank whose rows have none of the first tokens' targets takes the same factor
    dw = torch.cat([ar.vocab_loss_backward(dloss, x, w[a:b], target, lse, first=a, classes=size[2])[1] for a, b in ((0, 333), (333, size[2]))])
    exact, bound = oo.vocab_loss(x, w, target, dloss)["dw"]
    assert bool(((dw.cpu().double() - exact).abs() <= bound).all())


@pytest.mark.parametrize("tokens", [1, 300, 5000])
def test_no_token_leads(tokens):
    say("none", tokens)
    g = torch.Generator().manual_seed(4)
    x, w = torch.randn(tokens, 64, generator=g).bfloat16().cuda(), torch.randn(501, 64, generator=g).bfloat16().cuda()
    target, dloss = torch.full((tokens,), -1).cuda(), torch.full((tokens,), 0.3, device="cuda")
    for t in gradients(x, w, target, dloss):
        assert not t.any()
    for t in gradients(x, w, target.zero_(), dloss.zero_()):
        assert not t.any()
    dloss[-1] = math.inf
    dx, dw = gradients(x, w, target, dloss)
    assert not dx[:-1].any() and not torch.isfinite(dx[-1]).any() and not torch.isfinite(dw).any()


def test_a_graph_finds_it_again():
    """Replays with other tokens in front, in both ways of looking."""
    say("graphs")
    cases = []
    for size in ((300, 64, 1001, 20), (1300, 64, 1001, 20)):
        x, w, target, dloss = inputs(*size)
        lse = ar.vocab_loss(x, w, target)[1]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            ar.vocab_loss_backward(dloss, x, w, target, lse)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = ar.vocab_loss_backward(dloss, x, w, target, lse)
        cases.append((graph, got, (dloss, x, w, target, lse)))
    for turn in range(4):
        for graph, got, (dloss, x, w, target, lse) in cases:
            dloss.copy_(torch.where(target >= 0, (turn + 1) / COUNT, 0.0))
            target[:20 + 100 * turn] = -100
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(got, ar.vocab_loss_backward(dloss, x, w, target, lse)):
                assert torch.equal(a, b)
