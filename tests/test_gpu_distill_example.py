"""The example runs the vocabulary head's operators and the sparsifier together and learns."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_students_loss_falls():
    from paper_1911_08772_b200 import binding as gk, build
    build.build()
    gk.load()
    gk.gk_set_capacity(0)
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import distill_head
    finally:
        sys.path.pop(0)
    losses = distill_head.train(steps=30, rows=256, width=64, words=1003, k=16)
    assert all(math.isfinite(x) for x in losses)
    # a head of zeros: log of the vocabulary for the words, and no more than that for the pairs
    assert abs(losses[0] - math.log(1003)) <= math.log(1003)
    assert sum(losses[-3:]) / 3 < 0.9 * losses[0], losses
