"""The forward of the gated feed-forward block takes a workspace of what the call
uses, and a call that succeeds leaves no failure's code behind."""
from __future__ import annotations

import pytest
import torch

import paper_2603_11438_amd as ar
from gpu_helpers import say
from paper_2603_11438_amd import ops

pytestmark = pytest.mark.gpu

# in runs, nothing copied; copied, in one piece; and both
CALLS = [(1, 4096, 1408), (300, 999, 700), (5, 4357, 157)]


def operands(t, d, f):
    g = torch.Generator().manual_seed(t + d)
    rnd = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731
    return rnd(t, d), rnd(f, d), rnd(f, d)


@pytest.mark.parametrize("native", (True, False))
@pytest.mark.parametrize("t,d,f", CALLS)
def test_no_code_is_left_behind(monkeypatch, t, d, f, native):
    say(f"last error {t} x {d} x {f} native {native}")
    if not native:
        monkeypatch.setattr(ops, "_native_path", False)
    x, wg, wu = operands(t, d, f)
    with pytest.raises(ar.ARError):
        ar.gated_ffn(x.float(), wg.float(), wu.float())
    assert ar.ar_last_error() == ar.AR_ERR_UNSUPPORTED
    ar.gated_ffn(x, wg, wu)
    assert ar.ar_last_error() == ar.AR_ERR_UNSUPPORTED


@pytest.mark.parametrize("native", (True, False))
def test_runs_take_no_room_for_copies(monkeypatch, native):
    """1 x 4096 x 5632 in runs: fp32 sums of two projections for each of them, 32 at most."""
    if not native:
        monkeypatch.setattr(ops, "_native_path", False)
    x, wg, wu = operands(1, 4096, 5632)
    ar.gated_ffn(x, wg, wu)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    h = ar.gated_ffn(x, wg, wu)
    assert torch.cuda.max_memory_allocated() - before <= 32 * 2 * 5632 * 4 + h.numel() * 2 + 4096
