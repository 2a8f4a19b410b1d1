"""The example trains: norms, their gradients, clipping into the flat gradients and the compressed step together."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from paper_2008_11343_b200 import binding as B


@pytest.mark.parametrize("eight_bit", [False, True])
def test_the_example_learns_its_task(eight_bit):
    import train_block

    losses, norms, phase, launches = train_block.train(steps=60, eight_bit=eight_bit)
    assert all(math.isfinite(v) for v in losses + norms) and phase == B.PHASE_COMPRESSED and launches >= 60
    assert 0.5 * math.log(256) < losses[0] < 2.5 * math.log(256)               # random start, 256 tokens
    assert losses[39] < 0.5 * losses[0]                                       # warmup phase: Adam
    assert losses[-1] < 1.2 * losses[39]                                      # the compressed phase keeps it
    assert max(norms) > 1.0                                                   # something was clipped
