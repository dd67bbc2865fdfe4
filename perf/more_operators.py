"""The work that attention and the loss of a model shared by ranks are measured on.

A rank of a tensor-parallel program holds some of a block's heads and some rows
of the output projection's matrix.  Between two joins of the ranks it computes
attention on its heads, and at the model's end the softmax cross entropy over its
piece of the vocabulary.  These are the two families of cases:

  attn   attention over packed sequences of different lengths, grouped heads;
         forward, or forward and backward as in training
  loss   cross entropy of x W^T over a vocabulary, without keeping the logits;
         forward, over pieces of the vocabulary that are joined, or forward and
         backward as in training

With ``own`` false, ``run`` computes each in its plain form: elementary torch
operations in 32 bits, rounded once at the end.  With ``own`` true it makes the
calls of this repository's package.
"""
from __future__ import annotations

import math

import torch

own = False

# A case:
#   op       attn / loss
#   attn     lens_q, lens_k: queries and keys of each sequence; heads, kv_heads,
#            dim: of a head; causal: the last query sees all keys, each one before
#            it one key less; fused: q, k and v are column ranges of one tensor;
#            train: backward too
#   loss     tokens, dim, vocab; shards: pieces of the vocabulary, each a rank's;
#            train: backward too


def _attn(name, lens_q, lens_k, heads, kv_heads, dim, causal=True, train=False, fused=False):
    text = lambda lens: ",".join(str(n) for n in lens)  # noqa: E731
    return {"name": name, "op": "attn", "lens_q": text(lens_q), "lens_k": text(lens_k), "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "causal": causal, "train": train, "fused": fused}


def _loss(name, tokens, dim, vocab, train=False, shards=1):
    return {"name": name, "op": "loss", "tokens": tokens, "dim": dim, "vocab": vocab, "train": train, "shards": shards}


def listed():
    prompts, pieces = (8192, 5003, 2048, 1141), (777, 1, 2001, 64, 130)
    # lengths of a serving batch's caches, short ones and long ones
    caches = [160 + (k * 6151) % 15000 for k in range(32)]
    return [
        # One token of one sequence in a serving loop: all latency.
        _attn("attn_token", [1], [700], 32, 8, 128),
        # A step of a serving batch: a new token each, the caches are read once.
        _attn("attn_token_batch", [1] * 32, caches, 32, 8, 128),
        # A piece of a long prompt, whose beginning is in the cache already; a rank's few heads.
        _attn("attn_chunk", [512], [33000], 8, 1, 128),
        # A prefill of several prompts.
        _attn("attn_prompts", prompts, prompts, 32, 8, 128),
        # A training batch, a fused projection's result.
        _attn("attn_train_2x4k", [4096] * 2, [4096] * 2, 32, 8, 128, train=True, fused=True),
        # Packed documents, an odd head size, few heads.
        _attn("attn_train_ragged", pieces, pieces, 6, 2, 80, train=True),
        # Queries over another sequence's keys, no mask, as many key heads as heads.
        _attn("attn_train_cross", [1000, 333], [1500, 77], 12, 12, 64, causal=False, train=True),
        # One token's loss: the weights are read once.
        _loss("loss_token", 1, 4096, 32768),
        # Evaluation of a batch, the vocabulary split over four ranks.
        _loss("loss_fwd_shards", 4096, 2048, 65536, shards=4),
        # A training batch over a large vocabulary.
        _loss("loss_train_128k", 4096, 4096, 131072, train=True),
        # A small odd-sized model on a ragged batch.
        _loss("loss_train_ragged", 777, 1000, 5001, train=True),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, spread over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    """One more case: from one token to thousands, from one sequence to dozens, heads
    of 8 to 128 elements, vocabularies from a hundred to the listed largest, odd
    sizes among them, both directions."""
    if rng.random() < 0.6:
        kv_heads = rng.choice((1, 2, 3, 4, 8))
        heads = kv_heads * rng.choice((1, 1, 2, 3, 4, 8))
        dim = rng.choice((64, 128, 128, 8 * _spread(rng, 1, 16), _spread(rng, 8, 128)))
        kind = rng.choice(("token", "chunk", "self", "self", "cross"))
        train = kind != "token" and rng.random() < 0.6
        most = 1.2e12 / (14 if train else 4) / (heads * max(dim, 64))  # query-key pairs
        count = _spread(rng, 1, 48)
        if kind == "token":
            lens_k = [_spread(rng, 1, 16384) for _ in range(count)]
            return _unnamed(_attn("", [1] * count, lens_k, heads, kv_heads, dim))
        if kind == "chunk":
            count = min(count, 4)
            lens_q = [_spread(rng, 2, 1024) for _ in range(count)]
            past = max(1, min(32768, int(most / sum(lens_q)) - max(lens_q)))
            lens_k = [n + _spread(rng, 1, past) for n in lens_q]
        else:
            top = min(8192, int(math.sqrt(most / count)))
            lens_q = [_spread(rng, 1, max(2, top)) for _ in range(count)]
            lens_k = lens_q if kind == "self" else [_spread(rng, 1, max(2, top)) for _ in range(count)]
        causal = kind != "cross" and rng.random() < 0.85
        return _unnamed(_attn("", lens_q, lens_k, heads, kv_heads, dim, causal, train, kind == "self" and rng.random() < 0.5))
    train = rng.random() < 0.5
    dim, vocab = 8 * _spread(rng, 8, 640) - rng.choice((0, 0, 0, 3)), _spread(rng, 100, 131072)
    most = 4096 * 4096 * 131072 // (1 if train else 2)
    tokens = _spread(rng, 1, max(1, min(8192, most // (dim * vocab))))
    return _unnamed(_loss("", tokens, dim, vocab, train, 1 if train else rng.choice((1, 1, 2, 5))))


def _unnamed(case):
    del case["name"]
    return case


def _lens(text):
    return [int(n) for n in text.split(",")]


def _drawer(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(30011 + 7919 * seed)
    return g, lambda *shape: torch.randn(*shape, generator=g, device="cuda")


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _inputs(case, seed):
    g, randn = _drawer(seed)
    if case["op"] == "attn":
        tq, tk = sum(_lens(case["lens_q"])), sum(_lens(case["lens_k"]))
        h, hk, d = case["heads"], case["kv_heads"], case["dim"]
        # Some of a head's elements are far above the others, as after a projection.
        scale = torch.exp(0.4 * randn(d))
        if case["fused"]:
            qkv = randn(tq, h + 2 * hk, d)
            qkv[:, :h + hk] *= scale
            qkv = qkv.bfloat16()
            s = {"q": qkv[:, :h], "k": qkv[:, h:h + hk], "v": qkv[:, h + hk:]}
        else:
            s = {"q": (randn(tq, h, d) * scale).bfloat16(), "k": (randn(tk, hk, d) * scale).bfloat16(), "v": randn(tk, hk, d).bfloat16()}
        if case["train"]:
            s["do"] = (1e-2 * randn(tq, h, d)).bfloat16()
        return s
    t, d, v = case["tokens"], case["dim"], case["vocab"]
    # Logits of a few units; a target in sixteen is padding, and has no loss.
    s = {"x": randn(t, d).bfloat16(), "w": (2.0 / math.sqrt(d) * randn(v, d)).bfloat16(),
         "target": torch.randint(0, v, (t,), generator=g, device="cuda")}
    s["target"][torch.rand(t, generator=g, device="cuda") < 1 / 16] = -100
    if case["train"]:
        s["dloss"] = torch.full((t,), 1.0 / t, device="cuda")
    return s


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    if case["op"] == "attn":
        s["lens_q"], s["lens_k"] = _lens(case["lens_q"]), _lens(case["lens_k"])
        for key in ("q", "k"):
            s["starts_" + key] = torch.tensor(_starts(s["lens_" + key]), dtype=torch.int32, device="cuda")
    elif case["shards"] > 1:
        s["first"] = [r * case["vocab"] // case["shards"] for r in range(case["shards"] + 1)]
    return s


def _plain_attn(s):
    case = s["case"]
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    scale, group = 1 / math.sqrt(d), h // hk
    o, dq, dk, dv = (torch.zeros(s[key].shape, device=s[key].device) for key in ("q", "q", "k", "v"))
    q0 = k0 = 0
    for lq, lk in zip(s["lens_q"], s["lens_k"]):
        if lq == 0:
            k0 += lk
            continue
        # a key head and its group of heads at a time
        hidden = None
        if case["causal"]:
            hidden = torch.arange(lk, device=o.device)[None] > torch.arange(lq, device=o.device)[:, None] + (lk - lq)
        for j in range(hk):
            k, v = s["k"][k0:k0 + lk, j].float(), s["v"][k0:k0 + lk, j].float()
            heads = slice(j * group, (j + 1) * group)
            q = s["q"][q0:q0 + lq, heads].float().transpose(0, 1).contiguous()
            p = torch.matmul(q, k.t().contiguous()) * scale
            if hidden is not None:
                p = p.masked_fill(hidden, -math.inf)
            m = p.amax(-1, keepdim=True)
            p = torch.exp(p - torch.where(m == -math.inf, torch.zeros_like(m), m))
            total = p.sum(-1, keepdim=True)
            p = p / torch.where(total == 0, torch.ones_like(total), total)
            found = torch.matmul(p, v)
            o[q0:q0 + lq, heads] = found.transpose(0, 1)
            if case["train"]:
                do = s["do"][q0:q0 + lq, heads].float().transpose(0, 1).contiguous()
                ds = p * (torch.matmul(do, v.t().contiguous()) - (do * found).sum(-1, keepdim=True)) * scale
                dq[q0:q0 + lq, heads] = torch.matmul(ds, k).transpose(0, 1)
                dk[k0:k0 + lk, j] = torch.matmul(ds.view(-1, lk).t().contiguous(), q.view(-1, d))
                dv[k0:k0 + lk, j] = torch.matmul(p.view(-1, lk).t().contiguous(), do.view(-1, d))
        q0, k0 = q0 + lq, k0 + lk
    if not case["train"]:
        return {"o": o.bfloat16()}
    return {"o": o.bfloat16(), "dq": dq.bfloat16(), "dk": dk.bfloat16(), "dv": dv.bfloat16()}


def _plain_loss(s):
    x, w, target = s["x"].float(), s["w"].float(), s["target"]
    counts = target >= 0
    at = torch.where(counts, target, torch.zeros_like(target))[:, None]
    z = x @ w.t()
    m = z.amax(1, keepdim=True)
    picked = z.gather(1, at)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    loss = (torch.log(total) + m - picked)[:, 0]
    loss = torch.where(counts, loss, torch.zeros_like(loss))
    if not s["case"]["train"]:
        return {"loss": loss}
    dz = e / total
    dz.scatter_add_(1, at, torch.full_like(picked, -1.0))
    dz = dz * torch.where(counts, s["dloss"], torch.zeros_like(loss))[:, None]
    return {"loss": loss, "dx": (dz @ w).bfloat16(), "dw": (dz.t() @ x).bfloat16()}


_package = None


def _run_own(s):
    global _package
    if _package is None:
        import paper_2603_11438_amd as _package
    ar, case = _package, s["case"]
    if case["op"] == "attn":
        seqs = {"starts_q": s["starts_q"], "starts_k": s["starts_k"], "causal": case["causal"]}
        if not case["train"]:
            return {"o": ar.packed_attention(s["q"], s["k"], s["v"], **seqs)}
        o, lse = ar.packed_attention(s["q"], s["k"], s["v"], save=True, **seqs)
        dq, dk, dv = ar.packed_attention_backward(s["do"], s["q"], s["k"], s["v"], o, lse, **seqs)
        return {"o": o, "dq": dq, "dk": dk, "dv": dv}
    x, w, target = s["x"], s["w"], s["target"]
    if case["shards"] > 1:
        parts = torch.empty(case["shards"], 2, case["tokens"], device=x.device)
        for r, (a, b) in enumerate(zip(s["first"], s["first"][1:])):
            ar.vocab_loss_part(x, w[a:b], target, first=a, out=parts[r])
        return {"loss": ar.vocab_loss_join(parts, target, classes=case["vocab"])[0]}
    loss, lse = ar.vocab_loss(x, w, target)
    if not case["train"]:
        return {"loss": loss}
    dx, dw = ar.vocab_loss_backward(s["dloss"], x, w, target, lse)
    return {"loss": loss, "dx": dx, "dw": dw}


def run(state):
    if own:
        return _run_own(state)
    return {"attn": _plain_attn, "loss": _plain_loss}[state["case"]["op"]](state)


def _pairs(case):
    """Query-key pairs that the mask leaves."""
    n = 0
    for lq, lk in zip(_lens(case["lens_q"]), _lens(case["lens_k"])):
        if not case["causal"]:
            n += lq * lk
        else:  # query i sees i + lk - lq + 1 keys, none where that is below one
            seeing = min(lq, lk)
            n += seeing * lk - seeing * (seeing - 1) // 2
    return n


def work(case):
    if case["op"] == "attn":
        tq, tk, d = sum(_lens(case["lens_q"])), sum(_lens(case["lens_k"])), case["dim"]
        q, kv, pairs = tq * case["heads"] * d, tk * case["kv_heads"] * d, _pairs(case) * case["heads"]
        if case["train"]:  # q, k, v, do in; o and the three gradients out
            return {"bytes": 2 * (4 * q + 4 * kv), "flops": 14 * d * pairs}
        return {"bytes": 2 * (2 * q + 2 * kv), "flops": 4 * d * pairs}
    t, d, v = case["tokens"], case["dim"], case["vocab"]
    if case["train"]:  # x and w in, their gradients out
        return {"bytes": 4 * (t * d + v * d) + 16 * t, "flops": 6 * t * d * v}
    return {"bytes": 2 * (t * d + v * d) + 12 * t, "flops": 2 * t * d * v}


def exact(case, seed):
    """The operators' definitions in 64 bits; gradients by differentiating them."""
    s = _inputs(case, seed)
    if case["op"] == "attn":
        lens_q, lens_k, per = _lens(case["lens_q"]), _lens(case["lens_k"]), case["heads"] // case["kv_heads"]
        if (14 if case["train"] else 4) * _pairs(case) * case["heads"] * max(case["dim"], 64) > 2e13:
            return None
        out = {"o": torch.zeros_like(s["q"], dtype=torch.float64)}
        if case["train"]:
            out |= {"d" + n: torch.zeros_like(s[n], dtype=torch.float64) for n in "qkv"}
        for a, lq, b, lk in zip(_starts(lens_q), lens_q, _starts(lens_k), lens_k):
            if not lq or not lk:
                continue
            # queries that see no key have no part in it
            none = max(0, lq - lk) if case["causal"] else 0
            allowed = torch.ones(lq - none, lk, dtype=torch.bool, device="cuda")
            if case["causal"]:
                allowed = torch.tril(allowed, diagonal=lk - (lq - none))
            for h in range(case["heads"]):
                q, k, v = s["q"][a + none:a + lq, h].double(), s["k"][b:b + lk, h // per].double(), s["v"][b:b + lk, h // per].double()
                with torch.set_grad_enabled(case["train"]):
                    for t in (q, k, v):
                        t.requires_grad_(case["train"])
                    z = (q @ k.T) / case["dim"] ** 0.5
                    logp = z - torch.logsumexp(torch.where(allowed, z, -math.inf), 1)[:, None]
                    o = torch.where(allowed, logp, -math.inf).exp() @ v
                out["o"][a + none:a + lq, h] = o.detach()
                if case["train"]:
                    grads = torch.autograd.grad(o, (q, k, v), s["do"][a + none:a + lq, h].double())
                    out["dq"][a + none:a + lq, h] = grads[0]
                    out["dk"][b:b + lk, h // per] += grads[1]
                    out["dv"][b:b + lk, h // per] += grads[2]
        return out
    x, target = s["x"].double(), s["target"]
    counted = (target != -100).double()
    loss, dx = torch.zeros(case["tokens"], dtype=torch.float64, device="cuda"), torch.zeros_like(x)
    w = s["w"]
    dw = torch.zeros(w.shape, dtype=torch.float64, device="cuda") if case["train"] else None
    step = max(1, min(case["tokens"], (1 << 28) // case["vocab"]))
    w = w.double()
    for a in range(0, case["tokens"], step):
        z = x[a:a + step] @ w.T
        lse, rows = torch.logsumexp(z, 1), torch.arange(z.shape[0], device=z.device)
        hit = target[a:a + step].clamp(min=0)
        loss[a:a + step] = counted[a:a + step] * (lse - z[rows, hit])
        if case["train"]:
            z = torch.exp(z - lse[:, None])
            z[rows, hit] -= 1
            z *= (counted * s["dloss"].double())[a:a + step, None]
            dx[a:a + step] = z @ w
            dw += z.T @ x[a:a + step]
    return {"loss": loss, "dx": dx, "dw": dw} if case["train"] else {"loss": loss}
