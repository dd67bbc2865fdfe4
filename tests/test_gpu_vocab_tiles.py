"""Every tile of the vocabulary loss's products, ragged ends included, against its
definition in 64 bits at the sizes of loss_shapes.py, with the bounds that the oracle
derives for each element.  tests/test_vocab_cut.py holds the sizes to the tiles."""
from __future__ import annotations

import pytest

from gpu_helpers import say
from loss_shapes import SIZES
from test_gpu_vocab_loss import check_all, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_against_the_definition(size):
    say("loss", size)
    check_all(*inputs(*size, 21), device="cuda")
