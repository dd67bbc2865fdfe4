"""The operators and the collective together, attention to loss, as a shared model's
training step uses them, against the model in one piece in fp64 on the CPU.

Tolerance, of each result's norm: every tensor that is kept in bf16 on the way is off by
at most 2^-8 / sqrt(3) = 2.3e-3 of its norm.  Forward a dozen of them lie in a chain (qkv,
p, o, y, s1, x1, h, z and their partial sums), backward two dozen (dz of the loss, dx2, dz,
dh, dG and dU, dx1, dy, do, p, dz, dq, dk, dv, dx and their partial sums): together by
sqrt(36) * 2.3e-3 = 1.4e-2; 4e-2 leaves room for where the norms' and the softmaxes'
backward passes cancel."""
from __future__ import annotations

import math

import pytest
import torch

from gpu_helpers import say

pytestmark = pytest.mark.gpu

TOL = 4e-2


def plain(model, x, starts, target):
    """Losses and gradients of their mean in fp64, from the same weights and inputs."""
    wide = lambda t: t.detach().cpu().double().requires_grad_()  # noqa: E731
    h, hk, d = model.heads, model.kv_heads, model.head_dim
    x, ffn = wide(x), model.ffn
    w = {name: [wide(t) for t in ts] for name, ts in (("wqkv", model.wqkv), ("wo", model.wo), ("wg", ffn.wg), ("wu", ffn.wu), ("wd", ffn.wd),
                                                       ("vocab", model.vocab))}
    n = {name: wide(t) for name, t in (("post", model.post), ("pre", model.pre), ("ffn_post", ffn.post), ("ffn_pre", ffn.pre))}
    norm = lambda v, u: v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6) * u  # noqa: E731
    y = 0
    for r in range(model.ranks):
        qkv = (x @ w["wqkv"][r].T).view(-1, h + 2 * hk, d)
        out = []
        for i in range(h):
            q, k, v = qkv[:, i], qkv[:, h + i // (h // hk)], qkv[:, h + hk + i // (h // hk)]
            rows = []
            for a, b in zip(starts, starts[1:]):
                z = (q[a:b] @ k[a:b].T) / math.sqrt(d)
                rows.append(torch.softmax(z.masked_fill(torch.ones(b - a, b - a).triu(1).bool(), -math.inf), 1) @ v[a:b])
            rows.append(torch.zeros(x.shape[0] - starts[-1], d).double())
            out.append(torch.cat(rows))
        y = y + torch.stack(out, 1).reshape(x.shape[0], -1) @ w["wo"][r].T
    s1 = x + norm(y, n["post"])
    x1 = norm(s1, n["pre"])
    z = 0
    for r in range(model.ranks):
        g = x1 @ w["wg"][r].T
        z = z + (g * torch.sigmoid(g) * (x1 @ w["wu"][r].T)) @ w["wd"][r].T
    s2 = s1 + norm(z, n["ffn_post"])
    logits = norm(s2, n["ffn_pre"]) @ torch.cat(w["vocab"]).T
    loss = torch.nn.functional.cross_entropy(logits, target.cpu(), reduction="none", ignore_index=-100)
    mean = loss.sum() / (target >= 0).sum().cpu()
    mean.backward()
    grads = {name: torch.cat([t.grad.flatten() for t in ts]) for name, ts in w.items()} | {name: t.grad for name, t in n.items()}
    return {"loss": loss.detach(), "mean": mean.detach(), "s1": s1.detach(), "s2": s2.detach(), "dx": x.grad} | grads


@pytest.mark.parametrize("ranks,tokens,dim,heads,kv_heads,hidden,classes,head_dim,lens",
                         [(2, 150, 128, 8, 4, 256, 300, 64, [100, 1, 49]), (4, 97, 200, 4, 4, 264, 131, 40, [60, 30]), (1, 33, 72, 3, 1, 64, 50, 128, [33])])
def test_model(ranks, tokens, dim, heads, kv_heads, hidden, classes, head_dim, lens):
    from paper_2603_11438_amd.model_step import Model

    say("model", ranks, tokens, dim, heads, kv_heads, hidden, classes, head_dim, lens)
    model = Model(ranks, dim, heads, kv_heads, hidden, classes, head_dim=head_dim, seed=ranks)
    gen = torch.Generator().manual_seed(11)
    x = torch.randn(tokens, dim, generator=gen).cuda().bfloat16()
    target = torch.randint(0, classes, (tokens,), generator=gen)
    starts = [0]
    for n in lens:
        starts.append(starts[-1] + n)
    target[starts[-1]:] = -100  # padding behind the last sequence
    target[::7] = -100
    target = target.cuda()
    got = model.gradients(x, torch.tensor(starts, dtype=torch.int32).cuda(), target)
    for name, want in plain(model, x, starts, target).items():
        found = got[name]
        found = torch.cat([t.flatten() for t in found]) if isinstance(found, list) else found
        off = float((found.cpu().double() - want).norm() / want.norm())
        assert off <= TOL, f"{name} off by {off:.3g}"


def test_steps_run():
    from paper_2603_11438_amd import model_step

    losses = model_step.run(ranks=2, tokens=200, dim=128, heads=4, kv_heads=2, hidden=128, classes=333, steps=3, say=say)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)


def test_uneven_split_is_refused():
    from paper_2603_11438_amd.model_step import Model

    with pytest.raises(ValueError):
        Model(3, 64, 8, 4, 96, 100)
