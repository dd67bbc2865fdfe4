"""Every tile of the operators' products, ragged ends included: the gated
feed-forward block and its gradients, and orthogonalised updates, against 64 bits at
the sizes of gemm_shapes.py, with the tolerances of test_gpu_ffn.py and
test_gpu_ortho.py.  tests/test_gemm_cut.py holds the sizes to the tiles."""
from __future__ import annotations

import pytest
import torch

import paper_2603_11438_amd as ar
from gemm_shapes import FFN, ORTHO
from gpu_helpers import say
from test_gpu_ffn import check as check_ffn, inputs
from test_gpu_ortho import COEFS, tolerance

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,d,f", FFN)
def test_ffn(t, d, f):
    say(f"ffn {t} x {d} x {f}")
    check_ffn(*inputs(t, d, f, seed=5), "silu")


def orthogonalized(m):
    """The definition in 64 bits, on the GPU: the larger matrices take a CPU too long."""
    tall = m.shape[0] > m.shape[1]
    x = m.double()
    x = (x.t() if tall else x).contiguous()
    x = x / (torch.linalg.norm(x) + 1e-7)
    for _ in range(5):
        p = torch.matmul(x, x.t().contiguous())
        x = COEFS[0] * x + torch.matmul(COEFS[1] * p + COEFS[2] * torch.matmul(p, p), x)
    return x.t() if tall else x


@pytest.mark.parametrize("planes,m,n,batch", ORTHO)
def test_ortho(planes, m, n, batch):
    dtype = "bf16" if planes == 1 else "f32"
    say(f"ortho {batch} of {m} x {n} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(m + n)
    k = max(1, min(m, n) // 16)
    strong = torch.matmul(torch.randn(m, k, generator=g, device="cuda"), torch.randn(k, n, generator=g, device="cuda")) / k ** 0.5
    x = torch.stack([strong * (0.02 * b) + torch.randn(m, n, generator=g, device="cuda") for b in range(batch)])
    x = x.to(torch.bfloat16 if planes == 1 else torch.float32)
    x = x[0] if batch == 1 else x
    got = ar.orthogonalize(x)
    assert bool(torch.isfinite(got).all())
    for b in sorted({0, batch // 2, batch - 1}):
        one, have = (x, got) if batch == 1 else (x[b], got[b])
        want = orthogonalized(one)
        off = float((have.double() - want).norm() / want.norm())
        assert off <= tolerance(m, n, dtype), (b, off)
    if planes == 2:  # and no element is far off in a matrix that is right on the whole: errors spread like noise
        assert float((have.double() - want).abs().max()) <= 100 * tolerance(m, n, dtype) * float(want.norm()) / (m * n) ** 0.5
