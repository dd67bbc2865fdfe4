"""What attention's results hold where no sequence has a part in them: new results zeros,
the caller's own what they held."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2603_11438_amd as ar
from gpu_helpers import say

pytestmark = pytest.mark.gpu

TOKENS, HEADS, KV_HEADS, DIM = 400, 4, 2, 64
STARTS = {"padding": [37, 97, 167], "one": [100, 300], "no sequences": [0], "none either": [60]}


def on_gpu(at):
    return torch.tensor(at, dtype=torch.int32).cuda()


def draw(heads, seed):
    return torch.randn(TOKENS, heads, DIM, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def inputs():
    return draw(HEADS, 1), draw(KV_HEADS, 2), draw(KV_HEADS, 3), draw(HEADS, 4)


def leave_nan():
    """NaN in the memory that the next new tensors of the results' sizes get."""
    for heads, dtype in ((HEADS, torch.bfloat16), (KV_HEADS, torch.bfloat16)):
        kept = [torch.full((TOKENS, heads, DIM), math.nan, dtype=dtype, device="cuda") for _ in range(64)]
        del kept
    kept = [torch.full((HEADS, TOKENS), math.nan, device="cuda") for _ in range(64)]
    del kept


def outside(t, at, dim=0):
    """The tokens of no sequence."""
    return torch.cat([t.narrow(dim, 0, at[0]), t.narrow(dim, at[-1], TOKENS - at[-1])], dim)


@pytest.mark.parametrize("given", [(True, False, False), (False, True, True), (False, False, True), (False, False, False)], ids=str)
@pytest.mark.parametrize("name", list(STARTS))
def test_gradients_that_are_new_and_those_that_are_not(name, given):
    say("gradients", name, given)
    at, (q, k, v, do) = STARTS[name], inputs()
    kw = dict(starts_q=on_gpu(at))
    o, lse = ar.packed_attention(q, k, v, save=True, **kw)
    want = ar.packed_attention_backward(do, q, k, v, o, lse, **kw)
    out = tuple(torch.full_like(t, 7.0) if is_given else None for t, is_given in zip((q, k, v), given))
    leave_nan()
    got = ar.packed_attention_backward(do, q, k, v, o, lse, out=out, **kw)
    for g, mine, w in zip(got, out, want):
        assert mine is None or g is mine
        assert torch.equal(g[at[0]:at[-1]], w[at[0]:at[-1]])
        assert bool((outside(g, at) == (0.0 if mine is None else 7.0)).all())


@pytest.mark.parametrize("with_out", (False, True))
@pytest.mark.parametrize("name", list(STARTS))
def test_the_logarithms_that_are_kept(name, with_out):
    """lse is always a new result: zeros in tokens of no sequence, whatever is done to o there."""
    say("lse", name, with_out)
    at, (q, k, v, _) = STARTS[name], inputs()
    mine = torch.full_like(q, 7.0) if with_out else None
    leave_nan()
    o, lse = ar.packed_attention(q, k, v, starts_q=on_gpu(at), save=True, out=mine)
    assert mine is None or o is mine
    assert not outside(lse, at, 1).any()
    assert bool((outside(o, at) == (7.0 if with_out else 0.0)).all())
    if at[-1] > at[0]:
        part = [t[at[0]:at[-1]].clone() for t in (q, k, v)]
        want = ar.packed_attention(*part, starts_q=on_gpu([s - at[0] for s in at]), save=True)
        assert torch.equal(o[at[0]:at[-1]], want[0]) and torch.equal(lse[:, at[0]:at[-1]], want[1])
