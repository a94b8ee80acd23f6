"""Input and output of the low-precision block that share memory (no GPU needed: refused before any work)."""

import pytest
import torch

from paper_2608_09231_gb300 import lowbit


@pytest.mark.parametrize("a,b,shared", [
    (lambda x: x, lambda x: x, True),
    (lambda x: x[:4], lambda x: x[4:], False),
    (lambda x: x[:5], lambda x: x[4:], True),
    (lambda x: x[:, :8], lambda x: x[1:], True),
    (lambda x: x[:, :8], lambda x: x[:, 8:], False),
    (lambda x: x[:, :8], lambda x: x[:, 7:], True),
    (lambda x: x[:, 1:9], lambda x: x[1:, 9:], False),
    (lambda x: x[:0], lambda x: x, False),
    (lambda x: x, lambda x: x.clone(), False),
])
def test_overlap(a, b, shared):
    x = torch.zeros(8, 16)
    assert lowbit._overlap(a(x), b(x)) is shared and lowbit._overlap(b(x), a(x)) is shared


def test_a_step_in_place_is_refused():
    """In place, the change that is kept would be zero, and a reused step a copy."""
    block = lowbit.LowBitBlock.__new__(lowbit.LowBitBlock)
    h = torch.zeros(8, 128)
    with pytest.raises(ValueError, match="share memory"):
        block.full(h, h, [None] * 6)
    assert bool((h == 0).all())
