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
