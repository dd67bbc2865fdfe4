"""The gated feed-forward block on the GPU, forward and backward, against its
plain form in 64 bits (oracle/ops_oracle.py).

Tolerance.  u = 2^-24, r = 2^-8 (half a unit of the last of bf16's eight bits).
The projections add dim products in fp32: within (dim + 16) u of the sum of
their magnitudes.  h adds the activation's own arithmetic, (32 + |g|) u, and
one rounding, r.  The backward products take dG and dU rounded to bf16, r of
each, before they add their terms in fp32, and round their result: elementwise
that bounds every output by the sum of magnitudes; and since rounding errors
of different terms are independent, in the root mean square each of the two
roundings is at most r / sqrt(3), so large results are within 2 r / sqrt(6) in
norm, and 1.1 times that is asked."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2603_11438_amd as ar
from gpu_helpers import say
from oracle import ops_oracle as oo

pytestmark = pytest.mark.gpu

U, R = 2.0 ** -24, 2.0 ** -8


def rows_of(x, pad):
    if not pad:
        return x.contiguous()
    wide = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def inputs(t, d, f, pad=0, fused=False, seed=0):
    g = torch.Generator().manual_seed(seed + 31 * t + d + f)
    rnd = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731
    w = (torch.randn(2 * f, d, generator=g) / math.sqrt(d)).bfloat16().cuda()
    x, dh = rows_of(rnd(t, d), pad), rows_of(rnd(t, f), pad)
    wg, wu = (w[:f], w[f:]) if fused else (rows_of(w[:f].clone(), pad), rows_of(w[f:].clone(), pad))
    return x, wg, wu, dh


def within(got, want, tol, label):
    got = got.detach().cpu().double()
    assert bool(torch.isfinite(got).all()), label
    bad = (got - want).abs() > tol + 1e-30
    assert not bool(bad.any()), f"{label}: {int(bad.sum())} of {bad.numel()} off, worst {float(((got - want).abs() / (tol + 1e-30)).max()):.3g} x"


def check(x, wg, wu, dh, act):
    t, d = x.shape
    f = wg.shape[0]
    h, saved = ar.gated_ffn(x, wg, wu, act=act, save=True)
    e, g, u = oo.gated_ffn(x, wg, wu, act)
    X, G, W = x.cpu().double().abs(), wg.cpu().double().abs(), wu.cpu().double().abs()
    gm, um = X @ G.T, X @ W.T
    k = (d + 16) * U
    within(saved[0], g, k * gm, "G")
    within(saved[1], u, k * um, "U")
    a, da = oo.activation(g, act)
    within(h, e, 1.01 * R * e.abs() + 1.01 * (k * (da.abs() * gm * u.abs() + a.abs() * um + gm * um * k) + (32 + g.abs()) * U * e.abs())
           + U * g.abs() * u.abs(), "h")
    assert torch.equal(h, ar.gated_ffn(x, wg, wu, act=act)), "h with and without save"
    got = ar.gated_ffn_backward(dh, x, wg, wu, saved, act=act)
    dx, dwg, dwu, dg, du = oo.gated_ffn_backward(dh, x, wg, wu, act)
    # relu's slope jumps where G is within its error of zero
    edge = (g.abs() <= k * gm).double() * (u.abs() + 1) * dh.cpu().double().abs() if act == "relu" else 0
    # dG and dU off by their rounding and by the projections' errors, of slopes below 1.2 and curvatures below 1
    D = dh.cpu().double().abs()
    eg = 1.01 * R * dg.abs() + edge + 1.3 * D * k * (um + u.abs() * gm) + 64 * U * D * u.abs()
    eu = 1.01 * R * du.abs() + edge + 1.3 * D * k * gm + 64 * U * D * g.abs()
    mg, mu = dg.abs() + eg, du.abs() + eu
    within(got[0], dx, 1.01 * (R * dx.abs() + eg @ G + eu @ W + (2 * f + 16) * U * (mg @ G + mu @ W)), "dx")
    within(got[1], dwg, 1.01 * (R * dwg.abs() + eg.T @ X + (t + 16) * U * (mg.T @ X)), "dw_gate")
    within(got[2], dwu, 1.01 * (R * dwu.abs() + eu.T @ X + (t + 16) * U * (mu.T @ X)), "dw_up")
    if t * d >= 50000 and f * d >= 50000:
        for v, w, name in zip(got, (dx, dwg, dwu), ("dx", "dw_gate", "dw_up")):
            off = float((v.cpu().double() - w).norm() / w.norm())
            assert off < 1.1 * 2 * R / math.sqrt(6), (name, off)


SHAPES = [(1, 1, 1), (1, 64, 7), (5, 129, 3), (16, 64, 64), (17, 512, 200), (33, 65, 300), (64, 1000, 333), (65, 256, 129),
          (129, 320, 130), (300, 1000, 333), (520, 192, 700)]


@pytest.mark.parametrize("act", ("silu", "gelu", "relu"))
@pytest.mark.parametrize("t,d,f", SHAPES)
def test_against_plain(t, d, f, act):
    for pad, fused in ((0, False), (5, False), (0, True)):
        say(f"ffn {t} x {d} x {f} {act} pad {pad} fused {fused}")
        check(*inputs(t, d, f, pad, fused), act)


@pytest.mark.parametrize("t,d,f", [(2100, 512, 4100), (1, 2048, 5000), (40, 4096, 1024), (8, 8192, 96)])
def test_larger(t, d, f):
    """Sizes that take the large tiles, a k that is split, and long rows."""
    say(f"ffn {t} x {d} x {f}")
    check(*inputs(t, d, f), "silu")


def test_same_bits_every_time():
    x, wg, wu, dh = inputs(70, 320, 500)
    h, s = ar.gated_ffn(x, wg, wu, save=True)
    one = ar.gated_ffn_backward(dh, x, wg, wu, s)
    for _ in range(3):
        h2, s2 = ar.gated_ffn(x, wg, wu, save=True)
        two = ar.gated_ffn_backward(dh, x, wg, wu, s2)
        assert torch.equal(h, h2) and torch.equal(s, s2) and all(torch.equal(a, b) for a, b in zip(one, two))
    dx, none, none2 = ar.gated_ffn_backward(dh, x, wg, wu, s, need_dw=False)
    assert none is None and none2 is None and torch.equal(dx, one[0])
    none, dg, du = ar.gated_ffn_backward(dh, x, wg, wu, s, need_dx=False)
    assert none is None and torch.equal(dg, one[1]) and torch.equal(du, one[2])


def test_no_tokens():
    x, wg, wu, _ = inputs(4, 64, 32)
    h, s = ar.gated_ffn(x[:0], wg, wu, save=True)
    assert h.shape == (0, 32)
    dx, dg, du = ar.gated_ffn_backward(h, x[:0], wg, wu, s)
    assert dx.shape == (0, 64) and bool((dg == 0).all()) and bool((du == 0).all())


def test_bad_values_stay_in_their_row():
    """A NaN or infinity reaches its token's row of h and dx and no other."""
    x, wg, wu, dh = inputs(40, 128, 96)
    h = ar.gated_ffn(x, wg, wu)
    x[3, 5], x[9, 100] = float("nan"), float("inf")
    h2, s = ar.gated_ffn(x, wg, wu, save=True)
    keep = [i for i in range(40) if i not in (3, 9)]
    assert torch.equal(h[keep], h2[keep]) and bool(torch.isnan(h2[3]).all()) and not bool(torch.isfinite(h2[9]).any())
    dx = ar.gated_ffn_backward(dh, x, wg, wu, s, need_dw=False)[0]
    assert bool(torch.isfinite(dx[keep]).all()) and bool(torch.isnan(dx[3]).all())


def test_large_projections():
    """Projections far beyond what exp takes: h is g u, or zero."""
    x = torch.full((2, 64), 20.0, device="cuda").bfloat16()
    w = torch.full((4, 64), 1.0, device="cuda").bfloat16()
    w[2:] = -1
    for act in ("silu", "gelu", "relu"):
        h, s = ar.gated_ffn(x, w, w, act=act, save=True)
        assert bool((s[:, :, :2] == 1280).all()) and bool((h[:, :2].float() == 1280 * 1280).all()) and bool((h[:, 2:] == 0).all()), act
        dx = ar.gated_ffn_backward(torch.ones_like(h), x, w, w, s, act=act)[0]
        assert bool((dx.float() == 2 * 2 * 1280).all()), act


def test_stream_out_and_leading_dimensions():
    x, wg, wu, dh = inputs(24, 128, 64)
    h = ar.gated_ffn(x, wg, wu)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    wide = torch.zeros(24, 200, dtype=torch.bfloat16, device="cuda")
    st.wait_stream(torch.cuda.current_stream())
    got = ar.gated_ffn(x.view(2, 12, 128), wg, wu, out=wide[:, 100:164], stream=st)
    st.synchronize()
    assert torch.equal(got, h) and bool((wide[:, :100] == 0).all()) and bool((wide[:, 164:] == 0).all())


def test_graph_replays():
    x, wg, wu, dh = inputs(130, 192, 260)

    def work():
        h, s = ar.gated_ffn(x, wg, wu, save=True)
        return (h, *ar.gated_ffn_backward(dh, x, wg, wu, s))

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for k in range(4):
        x.copy_(inputs(130, 192, 260, seed=50 + k)[0])
        want = work()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


def test_backward_against_differences():
    """The change of sum(dh * h) along a direction, by differences of the fp32
    projections of forward calls; steps are exact in bf16.  The gradient is off
    by 2 r of the magnitudes at most; what the difference itself is off by its
    step is taken from the 64-bit form."""
    t, d, f, step = 24, 64, 48, 2.0 ** -5
    g = torch.Generator().manual_seed(3)
    grid = lambda *s: (torch.randint(-8, 9, s, generator=g).float() / 8).bfloat16().cuda()  # noqa: E731
    v = {"x": grid(t, d), "wg": grid(f, d) / 4, "wu": grid(f, d) / 4}
    dh = grid(t, f)

    def loss(u, plain):
        if plain:
            return float((dh.cpu().double() * oo.gated_ffn(u["x"], u["wg"], u["wu"])[0]).sum())
        _, s = ar.gated_ffn(u["x"], u["wg"], u["wu"], save=True)
        s = s.cpu().double()
        return float((dh.cpu().double() * oo.activation(s[0], "silu")[0] * s[1]).sum())

    _, s = ar.gated_ffn(v["x"], v["wg"], v["wu"], save=True)
    got = dict(zip(("x", "wg", "wu"), ar.gated_ffn_backward(dh, v["x"], v["wg"], v["wu"], s)))
    ref = dict(zip(("x", "wg", "wu"), oo.gated_ffn_backward(dh, v["x"], v["wg"], v["wu"])))
    for name in v:
        e = torch.randint(-1, 2, v[name].shape, generator=g).float().bfloat16().cuda() * (1 if name == "x" else 0.25)
        up, down = {**v, name: v[name] + step * e}, {**v, name: v[name] - step * e}
        fd = (loss(up, False) - loss(down, False)) / (2 * step)
        ref_an = float((ref[name] * e.cpu().double()).sum())
        off = abs((loss(up, True) - loss(down, True)) / (2 * step) - ref_an)
        an = float((got[name].cpu().double() * e.cpu().double()).sum())
        assert abs(fd - an) <= off + 2 * R * float((ref[name].abs() * e.cpu().double().abs()).sum()) + 1e-3, (name, fd, an, off)


# Few tiles: k is split and its runs joined; long and short k, ragged ends, one
# token to several tiles of them, and operands that have to be laid out.
@pytest.mark.parametrize("t,d,f,pad", [(1, 4096, 1408, 0), (5, 4357, 157, 0), (64, 1000, 64, 0), (64, 2056, 130, 8), (65, 4096, 130, 0),
                                       (160, 4488, 184, 0), (300, 1999, 61, 3), (747, 2048, 581, 0), (33, 128, 8, 0), (200, 192, 72, 0)])
def test_forward_of_narrow_shares(t, d, f, pad):
    for act in ("silu", "relu"):
        say(f"ffn forward {t} x {d} x {f} {act} pad {pad}")
        x, wg, wu, _ = inputs(t, d, f, pad, seed=3)
        e, g, u = oo.gated_ffn(x, wg, wu, act)
        X, G, W = x.cpu().double().abs(), wg.cpu().double().abs(), wu.cpu().double().abs()
        gm, um = X @ G.T, X @ W.T
        k = (d + 16) * U  # a split adds its runs one after another: no more terms in a row than one sum has
        h, saved = ar.gated_ffn(x, wg, wu, act=act, save=True)
        within(saved[0], g, k * gm, "G")
        within(saved[1], u, k * um, "U")
        # |act'| is below 1.13, |act(g)| at most |g|
        tol = 1.13 * k * gm * (u.abs() + k * um) + k * um * g.abs() + (32 + g.abs()) * U * (g * u).abs() + R * e.abs() * 1.01
        within(h, e, tol, "h")
        assert torch.equal(ar.gated_ffn(x, wg, wu, act=act), h)
        out = torch.full((t, f + 5), 7.0, dtype=torch.bfloat16, device="cuda")
        ar.gated_ffn(x, wg, wu, act=act, out=out[:, :f])
        assert torch.equal(out[:, :f], h) and bool((out[:, f:] == 7).all())


def test_narrow_share_graph_replays():
    x, wg, wu, _ = inputs(8, 4096, 256)
    ar.gated_ffn(x, wg, wu)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ar.gated_ffn(x, wg, wu)
    for k in range(4):
        x.copy_(inputs(8, 4096, 256, seed=50 + k)[0])
        want = ar.gated_ffn(x, wg, wu)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want), k
