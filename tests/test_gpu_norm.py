"""The residual norm on the GPU, forward and backward, against its plain form
in 64 bits (oracle/ops_oracle.py).

Tolerance.  u = 2^-24.  A row's sum of squares adds at most cols / 512 + 64
terms one after another in one thread, and six and up to sixteen partial sums
after that; its relative error is below that count times u, half of it in the
norm.  The handful of products around it adds a few u.  So an output is within
(48 + cols / 512) u of the sum of magnitudes that meet in it, twice that for
the backward pass, which takes two norms and one more sum; a parameter's
gradient also adds its rows, fewer than rows of them one after another.  bf16
outputs add half a unit of the last of their eight bits, at most 2^-8 of the value."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2603_11438_amd as ar
from gpu_helpers import say
from oracle import ops_oracle as oo

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


def near(got, want, mag, k, dtype, label):
    got, want = got.detach().cpu().double().reshape(want.shape), want
    tol = k * U * mag + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0) + 1e-37
    if dtype == "bf16":
        tol = tol * 1.01  # the value that is rounded is itself off by the first term
    bad = (got - want).abs() > tol
    assert not bool(bad.any()), f"{label}: {int(bad.sum())} of {bad.numel()} off, worst {float(((got - want).abs() / tol).max()):.3g} x the tolerance"
    assert bool(torch.isfinite(got).all()), label


def rows_of(x, pad):
    if not pad:
        return x.contiguous()
    wide = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def inputs(t, d, dtype, param, groups, pad, seed):
    g = torch.Generator().manual_seed(seed)
    dt, pt = TORCH[dtype], TORCH[param]
    rnd = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    mk = lambda x: rows_of(x.to(dt).cuda(), pad)  # noqa: E731
    v = {"y": mk(rnd(t, d) * torch.exp(rnd(t, 1))), "residual": mk(2 * rnd(t, d)), "ds": mk(rnd(t, d)), "dx": mk(rnd(t, d)),
         "w1": (1 + 0.2 * rnd(d)).to(pt).cuda(), "w2": (1 + 0.2 * rnd(d)).to(pt).cuda(), "gate": None}
    if groups:
        v["gate"] = rnd(groups, d).to(pt).cuda()
    if t > 2:
        v["y"][t // 2] = 0  # a row whose norm is eps alone
    return v


SHAPES = [(1, 1), (1, 7), (3, 64), (5, 513), (64, 1000), (300, 2501), (257, 4096), (2, 8192), (520, 1024), (300, 8200),
          (3, 40001), (1030, 96)]


@pytest.mark.parametrize("dtype,param", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("t,d", SHAPES)
def test_forward_and_backward(t, d, dtype, param):
    groups = {1: 1, 64: 16, 300: 300, 520: 5, 1030: 515, 257: 1}.get(t, 0)
    for pad in (0, 3):
        say(f"norm {t} x {d} {dtype} {param} gate rows {groups} pad {pad}")
        v = inputs(t, d, dtype, param, groups, pad, t * 7 + d)
        kw = dict(post_weight=v["w1"], pre_weight=v["w2"], gate=v["gate"], alpha=0.75, eps=EPS)
        ref = (v["w1"], v["w2"], v["gate"], 0.75, EPS)
        s, x = ar.residual_norm(v["y"], v["residual"], **kw)
        es, ex, ms, mx = oo.residual_norm(v["y"], v["residual"], *ref)
        k = 48 + d / 512
        near(s, es, ms, k, dtype, "s")
        near(x, ex, mx, 2 * k, dtype, "x")
        got = ar.residual_norm_backward(v["y"], v["residual"], v["ds"], v["dx"], **kw)
        want = oo.residual_norm_backward(v["y"], v["residual"], v["ds"], v["dx"], *ref)
        assert set(got) == set(want) - (set() if groups else {"dgate"})
        for name, val in got.items():
            sums = name in ("dgate", "dpost_weight", "dpre_weight")
            near(val, *want[name], 2 * k + (t if sums else 0), param if sums else dtype, name)


@pytest.mark.parametrize("post,pre", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("d", (200, 20001))
def test_norms_switched_off(post, pre, d):
    t, v = 37, inputs(37, d, "f32", "f32", 1, 0, 5)
    kw = dict(gate=v["gate"], alpha=-1.5, eps=EPS, post=post, pre=pre)
    w1, w2 = v["w1"] if post else None, v["w2"] if pre else None
    s, x = ar.residual_norm(v["y"], v["residual"], post_weight=w1, pre_weight=w2, **kw)
    es, ex, ms, mx = oo.residual_norm(v["y"], v["residual"], w1, w2, v["gate"], -1.5, EPS, post, pre)
    k = 48 + d / 512
    near(s, es, ms, k, "f32", "s")
    assert (x is None) == (not pre)
    if pre:
        near(x, ex, mx, 2 * k, "f32", "x")
    got = ar.residual_norm_backward(v["y"], v["residual"], None, v["dx"] if pre else None, post_weight=w1, pre_weight=w2, **kw)
    want = oo.residual_norm_backward(v["y"], v["residual"], None, v["dx"] if pre else None, w1, w2, v["gate"], -1.5, EPS, post, pre)
    for name, val in got.items():
        near(val, *want[name], 2 * k + t, "f32", name)


@pytest.mark.parametrize("d", (512, 20001))
def test_in_place_and_repeats(d):
    """Outputs in the inputs' place, and the same bits from every call."""
    v = inputs(65, d, "bf16", "f32", 5, 0, 9)
    kw = dict(post_weight=v["w1"], pre_weight=v["w2"], gate=v["gate"], eps=EPS)
    s, x = ar.residual_norm(v["y"], v["residual"], **kw)
    y2, r2 = v["y"].clone(), v["residual"].clone()
    a, b = ar.residual_norm(y2, r2, out=(r2, y2), **kw)
    assert a is r2 and b is y2 and torch.equal(a, s) and torch.equal(b, x)
    one = ar.residual_norm_backward(v["y"], s, v["ds"], v["dx"], **kw)
    ds, dx = v["ds"].clone(), v["dx"].clone()
    two = ar.residual_norm_backward(v["y"], s, ds, dx, out=(dx, ds), **kw)
    assert two["dy"] is dx and all(torch.equal(one[k], two[k]) for k in one)
    few = ar.residual_norm_backward(v["y"], s, v["ds"], v["dx"], param_grads=False, **kw)
    assert set(few) == {"dy", "dresidual"} and torch.equal(few["dy"], one["dy"])


def test_columns_of_one_buffer():
    """Results beside their inputs in the same rows."""
    v = inputs(40, 96, "f32", "f32", 0, 0, 11)
    wide = torch.zeros(40, 384, device="cuda")
    parts = [wide[:, i * 96:(i + 1) * 96] for i in range(4)]
    parts[0].copy_(v["y"]), parts[1].copy_(v["residual"])
    s, x = ar.residual_norm(parts[0], parts[1], eps=EPS, out=(parts[2], parts[3]))
    es, ex = ar.residual_norm(v["y"], v["residual"], eps=EPS)
    assert torch.equal(s, es) and torch.equal(x, ex)


def test_bad_values_stay_in_their_row():
    v = inputs(6, 300, "f32", "f32", 0, 0, 13)
    good = ar.residual_norm(v["y"], v["residual"], eps=EPS)
    v["y"][2, 17], v["residual"][4, 0] = float("nan"), float("inf")
    s, x = ar.residual_norm(v["y"], v["residual"], eps=EPS)
    keep = [0, 1, 3, 5]
    assert torch.equal(s[keep], good[0][keep]) and torch.equal(x[keep], good[1][keep])
    assert bool(torch.isnan(s[2]).all()) and bool(torch.isnan(x[2]).all())
    assert float(s[4, 0]) == float("inf") and bool(torch.isnan(x[4, 0])) and bool((x[4, 1:] == 0).all())


def test_no_rows():
    e = torch.empty(0, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    s, x = ar.residual_norm(e, e, post_weight=w)
    assert s.shape == x.shape == (0, 64)
    g = ar.residual_norm_backward(e, e, e, e, post_weight=w, pre_weight=w)
    assert bool((g["dpost_weight"] == 0).all()) and bool((g["dpre_weight"] == 0).all())


def test_stream_and_leading_dimensions():
    v = inputs(24, 160, "bf16", "bf16", 4, 0, 15)
    kw = dict(post_weight=v["w1"], gate=v["gate"], eps=EPS)
    s, x = ar.residual_norm(v["y"], v["residual"], **kw)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    s3, x3 = ar.residual_norm(v["y"].view(4, 6, 160), v["residual"].view(4, 6, 160), stream=st, **kw)
    st.synchronize()
    assert s3.shape == (4, 6, 160) and torch.equal(s3.view(24, 160), s) and torch.equal(x3.view(24, 160), x)


def test_graph_replays():
    v = inputs(50, 640, "bf16", "f32", 5, 0, 17)
    kw = dict(post_weight=v["w1"], pre_weight=v["w2"], gate=v["gate"], eps=EPS)
    work = lambda: ar.residual_norm_backward(v["y"], v["residual"], v["ds"], v["dx"], **kw)  # noqa: E731
    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for k in range(4):
        v["y"].copy_(inputs(50, 640, "bf16", "f32", 5, 0, 100 + k)["y"])
        want = work()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want), k


def test_backward_against_differences():
    """The change of a loss along a direction, by differences of forward calls
    in fp32.  h = 2^-7: the third derivative's share is h^2 / 6 of a term of the
    loss' own size, 1e-5, and rounding gives 100 u of that size over h, 8e-4."""
    t, d, h = 9, 256, 2.0 ** -7
    v = inputs(t, d, "f32", "f32", 3, 0, 19)
    v["y"][t // 2] = 1
    g = torch.Generator().manual_seed(1)
    rnd = lambda x: torch.randn(x.shape, generator=g).cuda()  # noqa: E731
    names = {"y": "dy", "residual": "dresidual", "w1": "dpost_weight", "w2": "dpre_weight", "gate": "dgate"}

    def loss(u):
        s, x = ar.residual_norm(u["y"], u["residual"], post_weight=u["w1"], pre_weight=u["w2"], gate=u["gate"], alpha=0.5, eps=EPS)
        return float((s.double() * v["ds"].double()).sum() + (x.double() * v["dx"].double()).sum())

    s, _ = ar.residual_norm(v["y"], v["residual"], post_weight=v["w1"], pre_weight=v["w2"], gate=v["gate"], alpha=0.5, eps=EPS)
    got = ar.residual_norm_backward(v["y"], s, v["ds"], v["dx"], post_weight=v["w1"], pre_weight=v["w2"], gate=v["gate"], alpha=0.5, eps=EPS)
    size = float(v["ds"].double().norm() + v["dx"].double().norm()) * np.sqrt(d)
    for name, key in names.items():
        e = rnd(v[name])
        if name == "y":
            e = e * v["y"].norm(dim=1, keepdim=True) / e.norm(dim=1, keepdim=True)  # rows differ in scale
        up, down = dict(v), dict(v)
        up[name], down[name] = v[name] + h * e, v[name] - h * e
        fd = (loss(up) - loss(down)) / (2 * h)
        an = float((got[key].double() * e.double()).sum())
        assert abs(fd - an) < 1e-3 * size, (name, fd, an, size)


# Rows at and beside the widths where the backward pass gives up the next row,
# keeps its parameter gradients in LDS, or leaves a row in memory.
WIDE = [(d, dtype) for dtype, widths in (("f32", (4100, 6144, 6147, 8190, 8192, 8196, 12285, 12288, 12290)),
                                         ("bf16", (8196, 12279, 12288, 12290))) for d in widths]


@pytest.mark.parametrize("d,dtype", WIDE)
def test_wide_rows_backward(d, dtype):
    """More rows than workgroups, gate rows that end inside and between them:
    each output against 64 bits, and the same bits in its input's place."""
    t = 520
    for groups, param in ((0, "f32"), (5, dtype), (260, "bf16")):
        say(f"norm backward {t} x {d} {dtype} gate rows {groups}")
        v = inputs(t, d, dtype, param, groups, 3 if d % 2 else 0, d + groups)
        kw = dict(post_weight=v["w1"], pre_weight=v["w2"], gate=v["gate"], alpha=0.75, eps=EPS)
        got = ar.residual_norm_backward(v["y"], v["residual"], v["ds"], v["dx"], **kw)
        want = oo.residual_norm_backward(v["y"], v["residual"], v["ds"], v["dx"], v["w1"], v["w2"], v["gate"], 0.75, EPS)
        k = 48 + d / 512
        for name, val in got.items():
            sums = name in ("dgate", "dpost_weight", "dpre_weight")
            near(val, *want[name], 2 * k + (t if sums else 0), param if sums else dtype, name)
        two = ar.residual_norm_backward(v["y"], v["residual"], v["ds"], v["dx"], out=(v["dx"], v["ds"]), **kw)
        assert all(torch.equal(got[n], two[n]) for n in got)


@pytest.mark.parametrize("post,pre", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("d", (6000, 12288))
def test_wide_rows_norms_switched_off(post, pre, d):
    t, v = 300, inputs(300, d, "f32", "f32", 3, 0, 23)
    w1, w2, dx = v["w1"] if post else None, v["w2"] if pre else None, v["dx"] if pre else None
    got = ar.residual_norm_backward(v["y"], v["residual"], None, dx, post_weight=w1, pre_weight=w2, gate=v["gate"], alpha=-1.5, eps=EPS,
                                    post=post, pre=pre)
    want = oo.residual_norm_backward(v["y"], v["residual"], None, dx, w1, w2, v["gate"], -1.5, EPS, post, pre)
    for name, val in got.items():
        near(val, *want[name], 2 * (48 + d / 512) + t, "f32", name)


@pytest.mark.parametrize("shape", [(), (1, 2, 64)])
def test_gate_is_a_row_or_a_matrix(shape):
    y = torch.zeros(4, 64, device="cuda")
    with pytest.raises(ValueError, match="gate must be"):
        ar.residual_norm(y, y, gate=torch.ones(shape, device="cuda"))
    with pytest.raises(ValueError, match="gate must be"):
        ar.residual_norm_backward(y, y, None, y, gate=torch.ones(shape, device="cuda"))
