"""The example that runs the calls on histories together: it learns, and what it serves event by event is what it trained."""
import math
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.gpu
def test_train_serve_and_meta_step():
    import history_tower
    losses, off, meta = history_tower.run(steps=30, users=64, items=2000, say=lambda *a: None)
    assert abs(losses[0] - math.log(2)) < 0.05           # rows of 0.1: scores near zero
    assert losses[-1] < losses[0] - 0.02
    # states are rounded to bf16 (2^-8) where they are stored, in both; a vector is an average of them, rounded again, and the two
    # forward passes take their sums in other orders: a few roundings of the largest entry
    assert off < 4 * 2.0 ** -8
    assert math.isfinite(meta)
