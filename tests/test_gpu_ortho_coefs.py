"""The coefficients that orthogonalize takes."""
from __future__ import annotations

import pytest
import torch

import paper_2603_11438_amd as ar

pytestmark = pytest.mark.gpu

A, B = (3.4445, -4.7750, 2.0315), (1.875, -1.25, 0.375)


def test_forms():
    x = torch.randn(20, 30, generator=torch.Generator().manual_seed(0)).cuda()
    want = ar.orthogonalize(x, steps=2, coefs=[A, B])
    assert torch.equal(ar.orthogonalize(x, steps=2, coefs=(list(A), B)), want)
    assert torch.equal(ar.orthogonalize(x, steps=2, coefs=torch.tensor([A, B], dtype=torch.float64)), want)
    assert torch.equal(ar.orthogonalize(x, steps=2, coefs=A), ar.orthogonalize(x, steps=2, coefs=[A, A]))


@pytest.mark.parametrize("steps,coefs", [(2, [(1.0, -0.5), (0.1, 1.5), (-0.5, 0.1)]), (2, [A, B, A]), (3, [A, B]), (1, A[:2]), (2, [A, B[:2]]),
                                         (1, [(1.5,), (-0.5,), (0.1,)]), (0, A), (17, A)])
def test_refused(steps, coefs):
    x = torch.randn(20, 30, generator=torch.Generator().manual_seed(0)).cuda()
    with pytest.raises(ValueError, match="one \\(a, b, c\\)"):
        ar.orthogonalize(x, steps=steps, coefs=coefs)
