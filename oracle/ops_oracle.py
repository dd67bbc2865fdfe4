"""Plain 64-bit forms of the operators around the collectives, on the CPU, and
for each output the sum of the magnitudes that meet in it: what a rounding
error is measured against.  Test infrastructure; shares no code with the
package."""
from __future__ import annotations

import math

import torch


def _d(t):
    return None if t is None else t.detach().cpu().double()


def rms(v, eps):
    return torch.sqrt((v * v).mean(-1, keepdim=True) + eps)


def residual_norm(y, residual, w1=None, w2=None, gate=None, alpha=1.0, eps=1e-6, post=True, pre=True):
    """(s, x, magnitude of s, magnitude of x)."""
    y, r, w1, w2, gate = _d(y), _d(residual), _d(w1), _d(w2), _d(gate)
    t, d = y.shape
    w1 = torch.ones(d).double() if w1 is None else w1
    w2 = torch.ones(d).double() if w2 is None else w2
    g = torch.ones(t, d).double() if gate is None else gate.reshape(-1, d).repeat_interleave(t // gate.reshape(-1, d).shape[0], 0)
    n = y / rms(y, eps) * w1 if post else y
    s = alpha * r + g * n
    mag = abs(alpha) * r.abs() + (g * n).abs()
    if not pre:
        return s, None, mag, None
    k = rms(s, eps)
    # a change of s reaches x directly and through the norm
    through = (s / k).abs() * (mag * s.abs()).mean(-1, keepdim=True) / k ** 2
    return s, s / k * w2, mag, (mag / k + through) * w2.abs()


def residual_norm_backward(y, s, ds, dx, w1=None, w2=None, gate=None, alpha=1.0, eps=1e-6, post=True, pre=True):
    """{name: (gradient, magnitude)}."""
    y, s, ds, dx, w1, w2, gate = (_d(v) for v in (y, s, ds, dx, w1, w2, gate))
    t, d = y.shape
    w1 = torch.ones(d).double() if w1 is None else w1
    w2 = torch.ones(d).double() if w2 is None else w2
    k = 1 if gate is None else gate.reshape(-1, d).shape[0]
    g = torch.ones(t, d).double() if gate is None else gate.reshape(-1, d).repeat_interleave(t // k, 0)

    def back(v, q):
        r = 1 / rms(v, eps)
        return (r * (q - v * r * r * (q * v).mean(-1, keepdim=True)),
                r * (q.abs() + v.abs() * r * r * (q * v).abs().mean(-1, keepdim=True)))

    total, mag = torch.zeros_like(y), torch.zeros_like(y)
    out = {}
    if ds is not None:
        total, mag = total + ds, mag + ds.abs()
    if pre:
        b, m = back(s, dx * w2)
        total, mag = total + b, mag + m
        out["dpre_weight"] = ((dx * s / rms(s, eps)).sum(0), (dx * s / rms(s, eps)).abs().sum(0))
    out["dresidual"] = (alpha * total, abs(alpha) * mag)
    r1 = 1 / rms(y, eps) if post else torch.ones(t, 1).double()
    unit = y * r1
    dn, dn_mag = total * g, mag * g.abs()
    n, n_mag = unit * w1 if post else unit, (unit * w1).abs() if post else unit.abs()
    out["dgate"] = ((total * n).reshape(k, -1, d).sum(1), (mag * n_mag).reshape(k, -1, d).sum(1))
    if post:
        out["dpost_weight"] = ((dn * unit).sum(0), (dn_mag * unit.abs()).sum(0))
        dy = back(y, dn * w1)[0]
        q = dn_mag * w1.abs()
        out["dy"] = (dy, r1 * (q + y.abs() * r1 * r1 * (q * y.abs()).mean(-1, keepdim=True)))
    else:
        out["dy"] = (dn, dn_mag)
    return out


def activation(g, kind):
    """The activation and its derivative."""
    if kind == "relu":
        return g.clamp(min=0), (g > 0).double()
    if kind == "silu":
        p = torch.sigmoid(g)
        return g * p, p + g * p * (1 - p)
    k = math.sqrt(2 / math.pi)
    th = torch.tanh(k * (g + 0.044715 * g ** 3))
    return g * (1 + th) / 2, (1 + th) / 2 + g * (1 - th * th) * k * (1 + 3 * 0.044715 * g * g) / 2


def gated_ffn(x, wg, wu, act="silu"):
    x, wg, wu = _d(x), _d(wg), _d(wu)
    g, u = x @ wg.T, x @ wu.T
    return activation(g, act)[0] * u, g, u


def gated_ffn_backward(dh, x, wg, wu, act="silu"):
    """dx, dwg, dwu and the factors dG and dU."""
    dh, x, wg, wu = _d(dh), _d(x), _d(wg), _d(wu)
    g, u = x @ wg.T, x @ wu.T
    a, da = activation(g, act)
    dg, du = dh * u * da, dh * a
    return dg @ wg + du @ wu, dg.T @ x, du.T @ x, dg, du


def orthogonalize(m, coefs, eps=1e-7, scale=1.0):
    """coefs: (a, b, c) of each step."""
    m = _d(m)
    x = m.T if m.shape[0] > m.shape[1] else m
    x = x / (torch.sqrt((x * x).sum()) + eps)
    for a, b, c in coefs:
        p = x @ x.T
        x = a * x + (b * p + c * (p @ p)) @ x
    x = scale * x
    return x.T if m.shape[0] > m.shape[1] else x


# bf16's and fp32's largest relative rounding error, and the room left for what fp32
# sums and exponentials are off by.
U, U32 = 2.0 ** -8, 2.0 ** -24
ROOM = 2.0 ** -14
# What fp32 and bf16 leave out at their lower end: a p below 2^-126 is 0 there.  Fewer than
# 2^26 such terms, each times factors whose product is below 1, or fewer by as much, are
# off by less than this.
UNDER = 2.0 ** -100


def attention(q, k, v, starts_q, starts_k, causal=True, scale=None, do=None):
    """Attention over packed sequences, and with `do` its gradients: {name: (value,
    bound)}, with bounds of what an implementation may be off by that rounds p and dz to
    bf16 as operands, sums in fp32 and rounds results to bf16.

    o: rounding p moves o by U M at most, M = sum p |v|; rounding o by U |o|.
    dv: likewise with M = sum_i p |do|.
    dq, dk: rounding dz: U sum |dz| |k|; the result: U |dq|; delta is taken from the
    rounded o: off by |do| . E, with E the bound of o, through p."""
    q, k, v, do = (_d(t) for t in (q, k, v, do))
    h, group, dim = q.shape[1], q.shape[1] // k.shape[1], q.shape[2]
    scale = dim ** -0.5 if scale is None else scale
    out = {n: (torch.zeros_like(t), torch.zeros_like(t)) for n, t in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64)
    for a, b, c, d in zip(starts_q, starts_q[1:], starts_k, starts_k[1:]):
        lq, lk = b - a, d - c
        if lq == 0 or lk == 0:
            continue
        sees = torch.ones(lq, lk, dtype=torch.bool)
        if causal:
            sees = torch.arange(lk)[None] <= torch.arange(lq)[:, None] + lk - lq
        for n in range(h):
            qi, kj, vj = q[a:b, n], k[c:d, n // group], v[c:d, n // group]
            z = torch.where(sees, scale * (qi @ kj.T), -math.inf)
            most = z.amax(1, keepdim=True)
            e = torch.exp(z - torch.where(most == -math.inf, 0.0, most))
            total = e.sum(1, keepdim=True)
            p = e / torch.where(total == 0, 1.0, total)
            lse[0][a:b, n] = torch.where(total == 0, -math.inf, most + torch.log(total))[:, 0]
            lse[1][a:b, n] = (dim + 16) * U32 * scale * torch.where(sees, qi.abs() @ kj.abs().T, 0.0).amax(1) + 2.0 ** -19
            # what z is off by in fp32 is p's relative error
            room = ROOM + 4 * lse[1][a:b, n, None]
            o, mag = p @ vj, p @ vj.abs()
            off = (U * 1.01 + room) * mag + U * o.abs()
            out["o"][0][a:b, n], out["o"][1][a:b, n] = o, off
            if do is None:
                continue
            g = do[a:b, n]
            dp, dp_mag = g @ vj.T, g.abs() @ vj.abs().T
            dz = p * (dp - (g * o).sum(1, keepdim=True))
            dz_off = (U * 1.01 + room) * dz.abs() + room * p * (dp_mag + (g * o).abs().sum(1, keepdim=True)) + \
                p * (g.abs() * off).sum(1, keepdim=True)
            for name, where, value, bound in (
                    ("dq", (slice(a, b), n), scale * dz @ kj, scale * dz_off @ kj.abs()),
                    ("dk", (slice(c, d), n // group), scale * dz.T @ qi, scale * dz_off.T @ qi.abs()),
                    ("dv", (slice(c, d), n // group), p.T @ g, ((U * 1.01 + room) * p).T @ g.abs())):
                out[name][0][where] += value
                out[name][1][where] += bound
    out["o"] = out["o"][0], out["o"][1] + UNDER
    for name in ("dq", "dk", "dv"):  # a result's own rounding
        out[name] = out[name][0], out[name][1] * (1 + U) + U * out[name][0].abs() + UNDER
    return {**out, "lse": lse}


def vocab_loss(x, w, target, dloss=None, device="cpu", chunk=1 << 26):
    """Cross entropy over a vocabulary, and with `dloss` its gradients: {name: (value,
    bound)}, with bounds of what an implementation may be off by that sums in fp32, rounds
    dz to bf16 as an operand and the gradients once.

    z: (dim + 16) U32 sum |x| |w|, a sum's bound; lse and loss: that, and a few roundings of
    theirs; p: relative to itself what z and lse are off by; dz: U of itself and p's; sums of
    dz: n U32 of their magnitudes, and U of the result."""
    x, w, target = x.detach().to(device).double(), w.detach().to(device).double(), target.detach().to(device).long()
    (t, dim), v = x.shape, w.shape[0]
    new = lambda *s: torch.zeros(*s, dtype=torch.float64, device=device)  # noqa: E731
    out = {"loss": (new(t), new(t)), "lse": (new(t), new(t))}
    if dloss is not None:
        dloss = dloss.detach().to(device).double().expand(t)
        out |= {"dx": (new(t, dim), new(t, dim)), "dw": (new(v, dim), new(v, dim))}
    for a in range(0, t, max(1, chunk // v)):
        rows = slice(a, min(t, a + max(1, chunk // v)))
        z, mag = x[rows] @ w.T, x[rows].abs() @ w.T.abs()
        counts = (target[rows] >= 0) & (target[rows] < v)
        at = torch.where(counts, target[rows], 0)[:, None]
        top = z.amax(1, keepdim=True)
        lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
        z_off = (dim + 16) * U32 * mag.amax(1, keepdim=True)
        lse_off = z_off + 2.0 ** -20 + 4 * U32 * (lse.abs() + top.abs())
        picked = z.gather(1, at)
        out["lse"][0][rows], out["lse"][1][rows] = lse[:, 0], lse_off[:, 0]
        out["loss"][0][rows] = torch.where(counts, (lse - picked)[:, 0], 0.0)
        out["loss"][1][rows] = torch.where(counts, (lse_off + z_off + 4 * U32 * picked.abs())[:, 0], 0.0)
        if dloss is None:
            continue
        g = torch.where(counts, dloss[rows], 0.0)[:, None]
        p = torch.exp(z - lse)
        room = (ROOM + 2 * (z_off + lse_off)) * p
        dz = p.scatter_add(1, at, torch.full_like(picked, -1.0)) * g
        off = (U * 1.01 + max(v, t) * U32) * dz.abs() + room * g.abs()
        out["dx"][0][rows], out["dx"][1][rows] = dz @ w, off @ w.abs()
        out["dw"][0].add_(dz.T @ x[rows]), out["dw"][1].add_(off.T @ x[rows].abs())
    for name in ("dx", "dw"):
        if name in out:
            out[name] = out[name][0], out[name][1] * (1 + U) + U * out[name][0].abs() + UNDER
    return out
