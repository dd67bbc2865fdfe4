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


@pytest.mark.parametrize("dim", [64, 100])
@pytest.mark.parametrize("heads_first", (False, True))
def test_parts_whose_heads_take_turns(heads_first, dim):
    """(tokens, heads, 3, dim), its gradients laid out the same, o beside do; as in tensors of their own."""
    say("in turn", heads_first, dim)
    g = torch.Generator().manual_seed(9)

    def fused(parts, fill=None):
        shape = (3, 150, parts, dim) if heads_first else (150, 3, parts, dim)
        t = torch.randn(*shape, generator=g).bfloat16().cuda() if fill is None else torch.full(shape, fill, dtype=torch.bfloat16, device="cuda")
        t = t.transpose(0, 1) if heads_first else t
        return [t[:, :, n] for n in range(parts)]

    starts, (q, k, v), (do, mine) = on_gpu([0, 90, 150]), fused(3), fused(2)
    before = do.clone()
    grads = fused(3, math.nan)
    assert ar.packed_attention(q, k, v, starts_q=starts, out=mine) is mine
    o, lse = ar.packed_attention(q, k, v, starts_q=starts, save=True)
    ar.packed_attention_backward(do, q, k, v, mine, lse, starts_q=starts, out=grads)
    apart = [t.clone(memory_format=torch.contiguous_format) for t in (do, q, k, v)]
    assert torch.equal(do, before) and torch.equal(mine, o) and torch.equal(ar.packed_attention(*apart[1:], starts_q=starts), o)
    for a, b in zip(grads, ar.packed_attention_backward(*apart, o, lse, starts_q=starts)):
        assert torch.equal(a, b)
    pair = fused(2, math.nan)
    ar.packed_attention_backward(do, q, k, v, o, lse, starts_q=starts, out=(None, *pair))
    assert torch.equal(pair[0], grads[1]) and torch.equal(pair[1], grads[2])
    with pytest.raises(ar.ARError):
        ar.packed_attention_backward(do, q, k, v, o, lse, starts_q=starts, out=(pair[0], pair[0], pair[1]))
