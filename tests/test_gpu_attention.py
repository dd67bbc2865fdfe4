"""Attention over packed sequences on the GPU, against its definition in 64 bits on the
CPU, with the bounds that the oracle derives for each element."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2603_11438_amd as ar
from gpu_helpers import say
from oracle import ops_oracle as oo

pytestmark = pytest.mark.gpu


def starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def on_gpu(at):
    return torch.tensor(at, dtype=torch.int32).cuda()


def draw(shape, seed, spread=1.0):
    return (spread * torch.randn(*shape, generator=torch.Generator().manual_seed(seed))).bfloat16().cuda()


def check(got, want, bound, name):
    got = got.detach().cpu().double()
    off = (got - want).abs()
    same = got == want  # infinities too
    assert bool((same | (off <= bound)).all()), f"{name}: {float((off / (bound + 1e-300))[~same].max()):.3g} times its bound"


def check_all(q, k, v, do, sq, sk, causal=True, scale=None):
    want = oo.attention(q, k, v, sq, sk, causal, scale, do)
    kw = dict(starts_q=on_gpu(sq), starts_k=on_gpu(sk), causal=causal, scale=scale)
    o, lse = ar.packed_attention(q, k, v, save=True, **kw)
    check(o, *want["o"], "o")
    check(lse.t(), *want["lse"], "lse")
    for name, g in zip(("dq", "dk", "dv"), ar.packed_attention_backward(do, q, k, v, o, lse, **kw)):
        check(g, *want[name], name)


def inputs(sq, sk, heads, kv_heads, dim, seed=0, spread=1.0):
    return (draw((sq[-1], heads, dim), seed, spread), draw((sk[-1], kv_heads, dim), seed + 1, spread), draw((sk[-1], kv_heads, dim), seed + 2),
            draw((sq[-1], heads, dim), seed + 3))


CASES = [
    # lengths of queries and keys, heads, key heads, dim, causal
    ([1], [1], 1, 1, 64, True), ([1], [2], 2, 1, 8, True), ([2], [1], 2, 2, 16, True), ([5], [5], 1, 1, 1, True), ([31], [31], 2, 1, 128, True),
    ([32], [33], 4, 4, 64, True), ([64], [64], 1, 1, 128, False), ([65], [63], 3, 1, 96, True), ([127, 129], [128, 128], 2, 2, 128, True),
    ([128], [300], 2, 1, 40, False), ([257], [257], 4, 2, 128, True), ([300, 1, 77], [300, 1, 77], 6, 2, 80, True),
    ([0, 40, 0], [7, 70, 0], 4, 2, 64, True), ([9, 9], [0, 200], 5, 1, 33, False), ([70] * 3, [3, 64, 71], 7, 7, 120, True),
    ([1] * 130, [(11 * i) % 97 for i in range(130)], 8, 1, 64, True), ([3] * 70, [200] * 70, 4, 4, 24, False),
    ([1], [3000], 8, 2, 128, True), ([1], [1999], 16, 1, 64, True), ([20], [2500], 3, 3, 127, True), ([700], [90], 2, 1, 64, True),
]


# More tiles than the device takes at once: the forward pass takes 128 rows a tile, but for
# single tokens.
MANY = [
    ([1], [1], 1200, 1200, 128, True), ([9], [5], 1200, 1200, 1, True), ([33], [32], 1800, 600, 128, True), ([65], [63], 600, 300, 96, True),
    ([127, 129], [128, 128], 240, 120, 128, True), ([300, 1, 77], [300, 1, 77], 270, 90, 80, True), ([0, 40, 0], [7, 70, 0], 600, 300, 64, True),
    ([9, 9], [0, 200], 650, 650, 33, False), ([70] * 3, [3, 64, 71], 130, 130, 120, True), ([128], [700], 260, 260, 40, False),
    ([20], [150], 1101, 1101, 127, True), ([700], [4000], 16, 1, 128, True), ([1200], [6000], 16, 1, 64, False),
    ([600], [3000], 16, 1, 128, True), ([1] * 20, [60 * i for i in range(20)], 32, 16, 64, True), ([8] * 80, [40] * 80, 12, 12, 72, True),
]
# Some sequences of many rows among those of few, some keys more than one tile of them is worth.
MIXED = [
    ([100, 1, 1, 1, 1, 1], [100, 30, 1, 2000, 64, 65], 8, 2, 128, True), ([1, 1, 70, 0, 1], [300, 0, 500, 9, 33], 12, 2, 72, True),
    ([33], [33], 4, 4, 128, True), ([16, 16], [1000, 1001], 2, 1, 64, True), ([17, 16], [1000, 1001], 2, 1, 64, False),
    ([1], [31], 8, 1, 128, True), ([1] * 4, [127, 128, 129, 160], 8, 1, 128, True), ([1] * 4, [255, 256, 257, 513], 8, 1, 56, True),
    ([256], [9000], 8, 1, 16, True),
]


@pytest.mark.parametrize("case", CASES + MANY + MIXED, ids=str)
def test_against_the_definition(case):
    lq, lk, heads, kv_heads, dim, causal = case
    say("attention", case)
    sq, sk = starts(lq), starts(lk)
    check_all(*inputs(sq, sk, heads, kv_heads, dim), sq, sk, causal)


@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (80, 40)])
@pytest.mark.parametrize("scale", [1e-3, 1.0, 20.0])
def test_scales(scale, heads, kv_heads):
    """From nearly even weights to weights on one key alone."""
    say("scale", scale, heads)
    sq = starts([150, 60])
    check_all(*inputs(sq, sq, heads, kv_heads, 64, 9), sq, sq, True, scale)


@pytest.mark.parametrize("heads,kv_heads", [(2, 1), (50, 25)])
def test_a_maximum_that_keeps_rising_and_one_that_comes_first(heads, kv_heads):
    say("rising", heads)
    n, d = 400, 64
    for order in (1.0, -1.0):
        sq = starts([n])
        q, k, v, do = inputs(sq, sq, heads, kv_heads, d, 20)
        q[..., 0], k[..., 0] = 8.0, (order * torch.linspace(-40, 40, n)).bfloat16().cuda()[:, None]
        check_all(q, k, v, do, sq, sq, False)


def test_one_sequence_needs_no_starts():
    q, k, v, do = inputs([0, 90], [0, 90], 4, 2, 64, 5)
    kw = dict(starts_q=on_gpu([0, 90]))
    o, lse = ar.packed_attention(q, k, v, save=True, **kw)
    o2, lse2 = ar.packed_attention(q, k, v, save=True)
    assert torch.equal(o, o2) and torch.equal(lse, lse2) and torch.equal(ar.packed_attention(q, k, v), o)
    for a, b in zip(ar.packed_attention_backward(do, q, k, v, o, lse, **kw), ar.packed_attention_backward(do, q, k, v, o, lse)):
        assert torch.equal(a, b)


def layouts(t, name):
    """The same values with other strides."""
    n, h, d = t.shape
    if name == "heads first":
        x = torch.empty(h, n, d, dtype=t.dtype, device=t.device).transpose(0, 1)
    elif name == "unaligned":
        x = torch.empty(n * h * d + 3, dtype=t.dtype, device=t.device)[3:].view(n, h, d)
    elif name == "apart":
        x = torch.full((n, h + 1, d + 8), math.nan, dtype=t.dtype, device=t.device)[:, :h, :d]
    else:
        x = torch.full((n, 2 * h, d + 5), math.nan, dtype=t.dtype, device=t.device)[:, ::2, 2:d + 2]
    return x.copy_(t)


@pytest.mark.parametrize("name", ["heads first", "unaligned", "apart", "odd apart"])
@pytest.mark.parametrize("heads", [6, 270])
@pytest.mark.parametrize("dim", [64, 100, 128])
def test_layouts(name, dim, heads):
    say("layout", name, dim, heads)
    sq, sk = starts([70, 5]), starts([130, 5])
    q, k, v, do = inputs(sq, sk, heads, heads // 3, dim, 30)
    kw = dict(starts_q=on_gpu(sq), starts_k=on_gpu(sk))
    o, lse = ar.packed_attention(q, k, v, save=True, **kw)
    grads = ar.packed_attention_backward(do, q, k, v, o, lse, **kw)
    q2, k2, v2, do2, o2 = (layouts(t, name) for t in (q, k, v, do, o))
    out = layouts(torch.zeros_like(q), name)
    assert ar.packed_attention(q2, k2, v2, out=out, **kw) is out and torch.equal(out, o)
    outs = [layouts(torch.zeros_like(t), name) for t in (q, k, v)]
    for got in (ar.packed_attention_backward(do2, q2, k2, v2, o2, lse, **kw), ar.packed_attention_backward(do2, q2, k2, v2, o2, lse, out=outs, **kw)):
        for a, b in zip(got, grads):
            assert torch.equal(a, b)


def test_parts_of_one_tensor():
    """A fused projection's result, and the gradients written as it is laid out."""
    say("fused")
    sq, h, hk, d = starts([100, 33]), 4, 2, 64
    qkv, grads = draw((sq[-1], h + 2 * hk, d), 40), torch.full((sq[-1], h + 2 * hk, d), math.nan, dtype=torch.bfloat16, device="cuda")
    do = draw((sq[-1], h, d), 41)
    parts = lambda t: (t[:, :h], t[:, h:h + hk], t[:, h + hk:])  # noqa: E731
    kw = dict(starts_q=on_gpu(sq))
    o, lse = ar.packed_attention(*parts(qkv), save=True, **kw)
    ar.packed_attention_backward(do, *parts(qkv), o, lse, out=parts(grads), **kw)
    want = oo.attention(*parts(qkv), sq, sq, do=do)
    check(o, *want["o"], "o")
    for g, name in zip(parts(grads), ("dq", "dk", "dv")):
        check(g, *want[name], name)


@pytest.mark.parametrize("lens", [[60, 70], [1, 1]])
def test_tokens_of_no_sequence(lens):
    """Padding may hold anything, and is left as it was in `out`, and zeros in new results."""
    say("padding", lens)
    before, behind = 37, 300
    sq = [before + n for n in starts(lens)]
    total = sq[-1] + behind
    inside = slice(before, sq[-1])
    q, k, v, do = (torch.full((total, n, 64), math.nan, dtype=torch.bfloat16, device="cuda") for n in (4, 2, 2, 4))
    for t, x in zip((q, k, v, do), inputs(starts(lens), starts(lens), 4, 2, 64, 50)):
        t[inside] = x
    kw = dict(starts_q=on_gpu(sq))
    o, lse = ar.packed_attention(q, k, v, save=True, **kw)
    grads = ar.packed_attention_backward(do, q, k, v, o, lse, **kw)
    want = oo.attention(q[inside], k[inside], v[inside], starts(lens), starts(lens), do=do[inside])
    check(o[inside], *want["o"], "o")
    check(lse[:, inside].t(), *want["lse"], "lse")
    assert not lse[:, :before].any() and not lse[:, sq[-1]:].any()
    for t, name in zip((o, *grads), ("o", "dq", "dk", "dv")):
        check(t[inside], *want[name], name)
        assert not t[:before].any() and not t[sq[-1]:].any(), name
    outs = [torch.full_like(t, 7.0) for t in (o, *grads)]
    ar.packed_attention(q, k, v, out=outs[0], **kw)
    ar.packed_attention_backward(do, q, k, v, o, lse, out=outs[1:], **kw)
    for t, new in zip(outs, (o, *grads)):
        assert torch.equal(t[inside], new[inside])
        assert bool((t[:before] == 7).all()) and bool((t[sq[-1]:] == 7).all())


@pytest.mark.parametrize("dim,heads", [(128, 8), (36, 5), (64, 1)])
def test_much_padding(dim, heads):
    """Far more padding than tokens, in every result."""
    say("much padding", dim, heads)
    sq = [3000, 3050]
    x = torch.full((9001, heads, dim), math.nan, dtype=torch.bfloat16, device="cuda")
    x[3000:3050] = draw((50, heads, dim), 51)
    o, lse = ar.packed_attention(x, x, x, starts_q=on_gpu(sq), save=True)
    grads = ar.packed_attention_backward(x, x, x, x, o, lse, starts_q=on_gpu(sq))
    part = x[3000:3050]
    want = oo.attention(part, part, part, [0, 50], [0, 50], do=part)
    for t, name in zip((o, lse.t(), *grads), ("o", "lse", "dq", "dk", "dv")):
        check(t[3000:3050], *want[name], name)
        assert not t[:3000].any() and not t[3050:].any()


@pytest.mark.parametrize("heads,kv_heads", [(2, 1), (160, 80)])
def test_keys_behind_a_sequences_end_do_not_reach_it(heads, kv_heads):
    """The next sequence's infinities and NaN lie in the same tiles."""
    say("neighbours", heads)
    sq = starts([50, 60, 30])
    q, k, v, do = inputs(sq, sq, heads, kv_heads, 64, 60)
    kw = dict(starts_q=on_gpu(sq))
    o, lse = ar.packed_attention(q, k, v, save=True, **kw)
    grads = ar.packed_attention_backward(do, q, k, v, o, lse, **kw)
    for t in (q, k, v, do):
        t[50:110] = math.nan
        t[60:70] = math.inf
    o2, lse2 = ar.packed_attention(q, k, v, save=True, **kw)
    grads2 = ar.packed_attention_backward(do, q, k, v, o2, lse2, **kw)
    for a, b in zip((o, lse.t(), *grads), (o2, lse2.t(), *grads2)):
        assert torch.equal(a[:50], b[:50]) and torch.equal(a[110:], b[110:])


@pytest.mark.parametrize("heads", [2, 48])
def test_later_keys_do_not_reach_a_query(heads):
    say("causal", heads)
    q, k, v, _ = inputs([0, 500], [0, 500], heads, heads // 2, 128, 61)
    o = ar.packed_attention(q, k, v)
    for t in (q, k, v):
        t[300:] = draw(t[300:].shape, 62, 50.0)
    k[320:340], q[400:] = math.nan, math.inf
    assert torch.equal(ar.packed_attention(q, k, v)[:300], o[:300])


def test_no_sequences_and_no_tokens():
    q, k, v, _ = inputs([0, 5], [0, 9], 2, 1, 64)
    none = on_gpu([0])
    assert not ar.packed_attention(q, k, v, starts_q=none).any()
    o, lse = ar.packed_attention(q[:0], k, v, starts_q=on_gpu([0, 0]), starts_k=on_gpu([0, 9]), save=True)
    assert o.shape == (0, 2, 64)
    dq, dk, dv = ar.packed_attention_backward(q[:0], q[:0], k, v, o, lse, starts_q=on_gpu([0, 0]), starts_k=on_gpu([0, 9]))
    assert dq.shape == (0, 2, 64) and not dk.any() and not dv.any()
    o, lse = ar.packed_attention(q, k[:0], v[:0], starts_q=on_gpu([0, 5]), starts_k=on_gpu([0, 0]), save=True)
    assert not o.any() and bool((lse == -math.inf).all())
    dq, dk, dv = ar.packed_attention_backward(q, q, k[:0], v[:0], o, lse, starts_q=on_gpu([0, 5]), starts_k=on_gpu([0, 0]))
    assert not dq.any() and dk.shape == (0, 1, 64)


def test_what_is_not_needed():
    q, k, v, do = inputs([0, 90], [0, 90], 4, 2, 64, 70)
    o, lse = ar.packed_attention(q, k, v, save=True)
    dq, dk, dv = ar.packed_attention_backward(do, q, k, v, o, lse)
    a, none, none2 = ar.packed_attention_backward(do, q, k, v, o, lse, need_dkv=False)
    assert none is None and none2 is None and torch.equal(a, dq)
    none, b, c = ar.packed_attention_backward(do, q, k, v, o, lse, need_dq=False)
    assert none is None and torch.equal(b, dk) and torch.equal(c, dv)
    ws = torch.empty(ar.packed_attention_backward_workspace(90, 90, 4, 2, 64), dtype=torch.uint8, device="cuda")
    for x, y in zip(ar.packed_attention_backward(do, q, k, v, o, lse, workspace=ws), (dq, dk, dv)):
        assert torch.equal(x, y)


def test_starts_outside_of_the_tokens_touch_nothing():
    """Values past the tokens are their end; decreasing ones give nothing defined, inside the results alone."""
    say("starts")
    sq = starts([40, 50])
    q, k, v, do = inputs(sq, sq, 2, 2, 64, 80)
    o, lse = ar.packed_attention(q, k, v, save=True, starts_q=on_gpu(sq))
    far = on_gpu([-5, 40, 1 << 30])
    o2, lse2 = ar.packed_attention(q, k, v, save=True, starts_q=far)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    for a, b in zip(ar.packed_attention_backward(do, q, k, v, o, lse, starts_q=far), ar.packed_attention_backward(do, q, k, v, o, lse, starts_q=on_gpu(sq))):
        assert torch.equal(a, b)


def test_another_stream_and_repeats():
    say("streams")
    sq = starts([200, 77, 1])
    q, k, v, do = inputs(sq, sq, 6, 2, 128, 90)
    kw = dict(starts_q=on_gpu(sq))
    o, lse = ar.packed_attention(q, k, v, save=True, **kw)
    grads = ar.packed_attention_backward(do, q, k, v, o, lse, **kw)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        o2, lse2 = ar.packed_attention(q, k, v, save=True, stream=other, **kw)
        grads2 = ar.packed_attention_backward(do, q, k, v, o2, lse2, stream=other, **kw)
        other.synchronize()
        for a, b in zip((o, lse, *grads), (o2, lse2, *grads2)):
            assert torch.equal(a, b)


def test_graphs():
    """Two captured steps with workspaces of their own, replayed between eager work, with
    other values and other lengths in the same memory."""
    say("graphs")
    sq, sk = [0, 60, 200], [0, 300, 900]
    q, k, v, do = inputs(sq, sk, 4, 2, 64, 100)
    a, b = on_gpu(sq), on_gpu(sk)

    def step(causal):
        o, lse = ar.packed_attention(q, k, v, starts_q=a, starts_k=b, causal=causal, save=True)
        return (o, lse, *ar.packed_attention_backward(do, q, k, v, o, lse, starts_q=a, starts_k=b, causal=causal))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(True)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for causal in (True, False):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = step(causal)
        graphs.append((g, causal, got))
    for turn in range(4):
        q.copy_(draw(q.shape, 200 + turn))
        a.copy_(on_gpu([0, 60 + 30 * turn, 200])), b.copy_(on_gpu([0, 300 - 70 * turn, 900]))
        for g, causal, got in graphs:
            g.replay()
            torch.cuda.synchronize()
            for x, y in zip(got, step(causal)):
                assert torch.equal(x, y)


def test_offsets_past_32_bits():
    """A cache of more than 2^31 elements: the sequence lies at its end."""
    say("large offsets")
    tokens, hk, d = (1 << 31) // (8 * 128) + 500, 8, 128
    k, v = (torch.zeros(tokens, hk, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[-300:], v[-300:] = draw((300, hk, d), 110), draw((300, hk, d), 111)
    q = draw((3, 16, d), 112)
    got = ar.packed_attention(q, k, v, starts_q=on_gpu([0, 0, 3]), starts_k=on_gpu([0, tokens - 300, tokens]))
    want = ar.packed_attention(q, k[-300:].clone(), v[-300:].clone())
    wide = oo.attention(q, k[-300:], v[-300:], [0, 3], [0, 300])
    check(got, *wide["o"], "o")
    check(want, *wide["o"], "o")


def test_refusals():
    q, k, v, do = inputs([0, 8], [0, 8], 4, 2, 64)
    o, lse = ar.packed_attention(q, k, v, save=True)
    a = on_gpu([0, 8])
    bad = [
        (ValueError, lambda: ar.packed_attention(q, k[:, :1].expand(8, 3, 64), v)), (ValueError, lambda: ar.packed_attention(q, k, v[:, :1])),
        (ValueError, lambda: ar.packed_attention(q, k[..., :32], v)), (TypeError, lambda: ar.packed_attention(q, k.float(), v)),
        (ValueError, lambda: ar.packed_attention(q[0], k, v)), (ValueError, lambda: ar.packed_attention(q, k, v, starts_k=a)),
        (ValueError, lambda: ar.packed_attention(q, k, v, starts_q=a.cpu())), (TypeError, lambda: ar.packed_attention(q, k, v, starts_q=a.long())),
        (ValueError, lambda: ar.packed_attention(q, k, v, starts_q=a, starts_k=on_gpu([0, 4, 8]))),
        (ValueError, lambda: ar.packed_attention(q, k, v, out=o[:4])), (ar.ARError, lambda: ar.packed_attention(q, k, v, out=q)),
        (ar.ARError, lambda: ar.packed_attention(q, k, v, scale=0.0)), (ar.ARError, lambda: ar.packed_attention(q, k, v, scale=math.inf)),
        (ar.ARError, lambda: ar.packed_attention(q.float(), k.float(), v.float())), (ValueError, lambda: ar.packed_attention(q.cpu(), k, v)),
        (ar.ARError, lambda: ar.packed_attention(draw((4, 2, 136), 0), draw((4, 2, 136), 0), draw((4, 2, 136), 0))),
        (ValueError, lambda: ar.packed_attention(q.transpose(1, 2), k, v)), (ValueError, lambda: ar.packed_attention_backward(do, q, k, v, o, lse[:, :4])),
        (ValueError, lambda: ar.packed_attention_backward(do[:4], q, k, v, o, lse)),
        (ar.ARError, lambda: ar.packed_attention_backward(do, q, k, v, o, lse, out=(do, torch.empty_like(k), torch.empty_like(v)))),
        (ar.ARError, lambda: ar.packed_attention_backward(do, q, k, v, o, lse, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))),
    ]
    for n, (kind, call) in enumerate(bad):
        with pytest.raises(kind):
            call()
            say("not refused:", n)
