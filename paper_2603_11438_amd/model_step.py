"""Training steps of a small model that N simulated ranks share, attention to loss, to
show the operators around the collectives at work:

    python -m paper_2603_11438_amd.model_step [--ranks 2] [--tokens 512] [--dim 256] [--heads 8] [--kv-heads 4]
                                              [--hidden 512] [--classes 1000] [--sequences 3] [--steps 4]

The model has one layer over packed sequences of tokens, x: an embedding's output.
Each rank has some of the heads, of the feed-forward block's hidden columns and of the
vocabulary's rows (tensor parallelism), so each product back to `dim` is a partial sum:

    packed_attention on the rank's heads, and the product with its columns of Wo
    allreduce;  s1, x1 = residual_norm(y, x)
    gated_ffn on the rank's rows, and the product with its columns of Wd
    allreduce;  s2, x2 = residual_norm(z, s1)
    vocab_loss_part on the rank's rows of the vocabulary
    allreduce of the parts;  vocab_loss_join

and back by the *_backward functions, with an allreduce of each partial gradient of
the stream.  The products with Wqkv, Wo and Wd are torch's.  Prints the mean loss of
each step and the time of the last one.
"""
from __future__ import annotations

import argparse
import sys

from .layer_step import Block


class Model:
    """The layer's weights, split over `ranks`, bf16; the norms' weights on every rank."""

    def __init__(self, ranks: int, dim: int, heads: int, kv_heads: int, hidden: int, classes: int, head_dim: int = 64, device="cuda",
                 seed: int = 0):
        import torch

        if ranks < 1 or kv_heads % ranks or heads % kv_heads:
            raise ValueError("kv_heads must be a multiple of ranks, heads of kv_heads")
        self.ranks, self.dim, self.head_dim, self.classes = ranks, dim, head_dim, classes
        self.heads, self.kv_heads = heads // ranks, kv_heads // ranks
        self.ffn = Block(ranks, dim, hidden, device=device, seed=seed)
        gen = torch.Generator().manual_seed(seed + 1)

        def draw(rows, cols):
            return (torch.randn(rows, cols, generator=gen) / cols ** 0.5).to(torch.bfloat16).to(device)

        part = self.heads + 2 * self.kv_heads
        self.wqkv = [draw(part * head_dim, dim) for _ in range(ranks)]
        self.wo = [draw(dim, self.heads * head_dim) for _ in range(ranks)]
        self.first = [r * classes // ranks for r in range(ranks + 1)]
        self.vocab = [draw(b - a, dim) for a, b in zip(self.first, self.first[1:])]
        self.post, self.pre = (torch.ones(dim, device=device) for _ in range(2))  # of the norms behind attention

    def _parts(self, qkv):
        qkv = qkv.view(-1, self.heads + 2 * self.kv_heads, self.head_dim)
        return qkv[:, :self.heads], qkv[:, self.heads:self.heads + self.kv_heads], qkv[:, self.heads + self.kv_heads:]

    def gradients(self, x, starts, target) -> dict:
        """The tokens' losses, and the gradients of their mean.  Every rank holds the same
        x, starts and target; what only repeats on the other ranks is done once."""
        import torch

        from . import (allreduce, gated_ffn, gated_ffn_backward, packed_attention, packed_attention_backward, residual_norm,
                       residual_norm_backward, vocab_loss_backward, vocab_loss_join, vocab_loss_part)

        ranks, ffn, tokens = range(self.ranks), self.ffn, x.shape[0]
        qkv = [x @ self.wqkv[r].t() for r in ranks]
        o, kept = zip(*(packed_attention(*self._parts(qkv[r]), starts_q=starts, save=True) for r in ranks))
        ys = [o[r].view(tokens, -1) @ self.wo[r].t() for r in ranks]
        allreduce(ys)
        norm1, norm2 = dict(post_weight=self.post, pre_weight=self.pre), dict(post_weight=ffn.post, pre_weight=ffn.pre)
        s1, x1 = residual_norm(ys[0], x, **norm1)
        h, saved = zip(*(gated_ffn(x1, ffn.wg[r], ffn.wu[r], save=True) for r in ranks))
        zs = [h[r] @ ffn.wd[r].t() for r in ranks]
        allreduce(zs)
        s2, x2 = residual_norm(zs[0], s1, **norm2)
        # each rank fills its own part of a buffer of zeros, and the sum has them all
        parts = [torch.zeros(self.ranks, 2, tokens, device=x.device) for _ in ranks]
        for r in ranks:
            vocab_loss_part(x2, self.vocab[r], target, first=self.first[r], out=parts[r][r])
        flat = [p.view(-1) for p in parts]
        allreduce(flat)
        loss, lse = vocab_loss_join(parts[0], target, classes=self.classes)

        counted = ((target >= 0) & (target < self.classes)).sum().clamp(min=1)
        d_loss = (1.0 / counted).float().expand(tokens)
        dxs, d_vocab = zip(*(vocab_loss_backward(d_loss, x2, self.vocab[r], target, lse, first=self.first[r], classes=self.classes)
                             for r in ranks))
        dxs = list(dxs)
        allreduce(dxs)
        g2 = residual_norm_backward(zs[0], s2, None, dxs[0], **norm2)
        d_wd = [g2["dy"].t() @ h[r] for r in ranks]
        dxs, d_wg, d_wu = map(list, zip(*(gated_ffn_backward(g2["dy"] @ ffn.wd[r], x1, ffn.wg[r], ffn.wu[r], saved[r]) for r in ranks)))
        allreduce(dxs)
        g1 = residual_norm_backward(ys[0], s1, g2["dresidual"], dxs[0], **norm1)
        d_wo, d_wqkv, dxs = [], [], []
        for r in ranks:
            d_wo.append(g1["dy"].t() @ o[r].view(tokens, -1))
            d_qkv = torch.zeros_like(qkv[r])  # tokens of no sequence have no gradient
            packed_attention_backward((g1["dy"] @ self.wo[r]).view_as(o[r]), *self._parts(qkv[r]), o[r], kept[r], starts_q=starts,
                                      out=self._parts(d_qkv))
            d_wqkv.append(d_qkv.t() @ x)
            dxs.append(d_qkv @ self.wqkv[r])
        allreduce(dxs)
        return {"loss": loss, "mean": loss.sum() / counted, "s1": s1, "s2": s2, "dx": dxs[0] + g1["dresidual"], "wqkv": d_wqkv, "wo": d_wo,
                "wg": d_wg, "wu": d_wu, "wd": d_wd, "vocab": list(d_vocab), "post": g1["dpost_weight"], "pre": g1["dpre_weight"],
                "ffn_post": g2["dpost_weight"], "ffn_pre": g2["dpre_weight"]}

    def update(self, grads: dict, rate: float) -> None:
        """Takes each rank's matrices a step along its orthogonalised gradients, and the
        vocabulary along its plain ones."""
        from . import orthogonalize

        for weights, found in ((self.wqkv, grads["wqkv"]), (self.wo, grads["wo"]), (self.ffn.wg, grads["wg"]), (self.ffn.wu, grads["wu"]),
                               (self.ffn.wd, grads["wd"])):
            for w, d in zip(weights, found):
                w.add_(orthogonalize(d, scale=max(1.0, w.shape[0] / w.shape[1]) ** 0.5), alpha=-rate)
        for w, d in zip(self.vocab, grads["vocab"]):
            w.add_(d, alpha=-rate)


def run(ranks: int = 2, tokens: int = 512, dim: int = 256, heads: int = 8, kv_heads: int = 4, hidden: int = 512, classes: int = 1000,
        sequences: int = 3, steps: int = 4, rate: float = 0.02, seed: int = 0, say=print) -> list:
    """The mean losses of `steps` steps on random inputs, in sequences of different lengths."""
    import torch

    model = Model(ranks, dim, heads, kv_heads, hidden, classes, seed=seed)
    gen = torch.Generator().manual_seed(seed + 2)
    x = torch.randn(tokens, dim, generator=gen).cuda().bfloat16()
    target = torch.randint(0, classes, (tokens,), generator=gen).cuda()
    cuts = sorted(int(v) for v in torch.randint(0, tokens + 1, (max(0, sequences - 1),), generator=gen))
    starts = torch.tensor([0, *cuts, tokens], dtype=torch.int32).cuda()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    losses = []
    for step in range(steps):
        begin.record()
        grads = model.gradients(x, starts, target)
        model.update(grads, rate)
        end.record()
        losses.append(float(grads["mean"]))
        say(f"step {step}: loss {losses[-1]:.5f}")
    if steps:
        say(f"last step: {begin.elapsed_time(end):.3f} ms on the device, {ranks} ranks, {tokens} tokens of {dim}, {heads} heads over "
            f"{kv_heads}, hidden {hidden}, {classes} classes")
    return losses


def main(argv=None) -> int:
    ap = argparse.ArgumentParser(description="training steps of a small model shared by simulated ranks")
    for name, value in (("ranks", 2), ("tokens", 512), ("dim", 256), ("heads", 8), ("kv-heads", 4), ("hidden", 512), ("classes", 1000),
                        ("sequences", 3), ("steps", 4), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--rate", type=float, default=0.02, help="length of an update of each weight matrix")
    run(**vars(ap.parse_args(argv)))
    return 0


if __name__ == "__main__":
    sys.exit(main())
