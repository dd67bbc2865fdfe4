"""Training steps of one feed-forward block that N simulated ranks share, to show
the operators around the collectives at work:

    python -m paper_2603_11438_amd.layer_step [--ranks 4] [--tokens 512] [--dim 512] [--hidden 1024] [--steps 4]

The block is x -> s, out = residual + norm(f(x)), norm(s) with the gated
feed-forward f(x) = (act(x Wg^T) * (x Wu^T)) Wd^T.  Its hidden columns are split
over the ranks (tensor parallelism), so each rank's f is a partial sum:

    gated_ffn on the rank's rows of Wg and Wu, and the product with its columns of Wd
    allreduce of the partial sums
    residual_norm of the joined sum
    residual_norm_backward, the products with Wd, gated_ffn_backward
    allreduce of the partial dx
    orthogonalize of each rank's weight gradients, which are its own: the update

The products with Wd are torch's.  Prints the loss of each step, a mean square
distance to fixed targets, and the time of the last step.
"""
from __future__ import annotations

import argparse
import sys


class Block:
    """The block's weights, split over `ranks`, bf16; the norms' weights on every rank."""

    def __init__(self, ranks: int, dim: int, hidden: int, device="cuda", seed: int = 0, act: str = "silu"):
        import torch

        if ranks < 1 or hidden % ranks:
            raise ValueError("hidden must be a multiple of ranks")
        self.ranks, self.dim, self.part, self.act = ranks, dim, hidden // ranks, act
        gen = torch.Generator().manual_seed(seed)

        def draw(rows, cols):
            w = torch.randn(rows, cols, generator=gen) / cols ** 0.5
            return w.to(torch.bfloat16).to(device)

        wg, wu, wd = draw(hidden, dim), draw(hidden, dim), draw(dim, hidden)
        self.wg = [w.clone() for w in wg.chunk(ranks)]
        self.wu = [w.clone() for w in wu.chunk(ranks)]
        self.wd = [w.contiguous() for w in wd.chunk(ranks, dim=1)]
        self.post = torch.ones(dim, device=device)
        self.pre = torch.ones(dim, device=device)

    def gradients(self, x, residual, target, alpha: float = 1.0) -> dict:
        """Loss and gradients of mean((out - target)^2).  Every rank holds the
        same x, residual and target; what only repeats on the other ranks is
        done once."""
        import torch

        from . import allreduce, gated_ffn, gated_ffn_backward, residual_norm, residual_norm_backward

        ranks = range(self.ranks)
        h, saved = zip(*(gated_ffn(x, self.wg[r], self.wu[r], act=self.act, save=True) for r in ranks))
        ys = [h[r] @ self.wd[r].t() for r in ranks]
        allreduce(ys)
        y = ys[0]
        norm = dict(post_weight=self.post, pre_weight=self.pre, alpha=alpha)
        s, out = residual_norm(y, residual, **norm)
        off = out.float() - target
        d_out = (off * (2.0 / off.numel())).to(out.dtype)
        g = residual_norm_backward(y, s, None, d_out, **norm)
        dxs, dwg, dwu, dwd = [], [], [], []
        for r in ranks:
            dwd.append(g["dy"].t() @ h[r])
            dx, dg, du = gated_ffn_backward(g["dy"] @ self.wd[r], x, self.wg[r], self.wu[r], saved[r], act=self.act)
            dxs.append(dx), dwg.append(dg), dwu.append(du)
        allreduce(dxs)
        return {"loss": off.square().mean(), "out": out, "s": s, "dx": dxs[0], "dresidual": g["dresidual"],
                "dpost": g["dpost_weight"], "dpre": g["dpre_weight"], "dwg": dwg, "dwu": dwu, "dwd": dwd,
                "y": torch.stack(ys) if self.ranks > 1 else y[None]}

    def update(self, grads: dict, rate: float) -> None:
        """Takes each rank's weights a step along its orthogonalised gradients."""
        from . import orthogonalize

        for weights, found in ((self.wg, grads["dwg"]), (self.wu, grads["dwu"]), (self.wd, grads["dwd"])):
            for w, d in zip(weights, found):
                w.add_(orthogonalize(d, scale=max(1.0, w.shape[0] / w.shape[1]) ** 0.5), alpha=-rate)


def run(ranks: int = 4, tokens: int = 512, dim: int = 512, hidden: int = 1024, steps: int = 4, rate: float = 0.02,
        seed: int = 0, say=print) -> list:
    """The losses of `steps` steps on random inputs."""
    import torch

    block = Block(ranks, dim, hidden, seed=seed)
    gen = torch.Generator().manual_seed(seed + 1)
    x, residual, target = (torch.randn(tokens, dim, generator=gen).cuda() for _ in range(3))
    x, residual = x.bfloat16(), residual.bfloat16()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    losses = []
    for step in range(steps):
        begin.record()
        grads = block.gradients(x, residual, target)
        block.update(grads, rate)
        end.record()
        losses.append(float(grads["loss"]))
        say(f"step {step}: loss {losses[-1]:.5f}")
    if steps:
        say(f"last step: {begin.elapsed_time(end):.3f} ms on the device, {ranks} ranks, {tokens} x {dim}, hidden {hidden}")
    return losses


def main(argv=None) -> int:
    ap = argparse.ArgumentParser(description="training steps of a block shared by simulated ranks")
    for name, value in (("ranks", 4), ("tokens", 512), ("dim", 512), ("hidden", 1024), ("steps", 4), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--rate", type=float, default=0.02, help="length of an update of each weight matrix")
    run(**vars(ap.parse_args(argv)))
    return 0


if __name__ == "__main__":
    sys.exit(main())
