"""orthogonalize between column ranges of one buffer."""
from __future__ import annotations

import pytest
import torch

import paper_2603_11438_amd as ar
from gpu_helpers import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_columns_of_one_buffer(dtype):
    say("ortho columns of one buffer", dtype)
    g = torch.randn(3, 90, 150, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    want = ar.orthogonalize(g)
    wide = torch.zeros(90, 400, dtype=dtype, device="cuda")
    wide[:, :150] = g[0]
    got = ar.orthogonalize(wide[:, :150], out=wide[:, 200:350])
    assert torch.equal(got, ar.orthogonalize(g[0])) and torch.equal(wide[:, :150], g[0])
    assert bool((wide[:, 150:200] == 0).all()) and bool((wide[:, 350:] == 0).all())
    deep = torch.zeros(3, 90, 320, dtype=dtype, device="cuda")
    deep[:, :, :150] = g
    assert torch.equal(ar.orthogonalize(deep[:, :, :150], out=deep[:, :, 160:310]), want)
    side = torch.zeros(90, 3, 2, 160, dtype=dtype, device="cuda")  # in, out, in, out .. in the same rows
    side[:, :, 0, :150] = g.permute(1, 0, 2)
    places = side.permute(1, 2, 0, 3)[..., :150]
    assert torch.equal(ar.orthogonalize(places[:, 0], out=places[:, 1]), want)
    assert torch.equal(places[:, 0], g) and bool((side[..., 150:] == 0).all())
    with pytest.raises(ar.ARError):
        ar.orthogonalize(wide[:, :150], out=wide[:, 149:299])
