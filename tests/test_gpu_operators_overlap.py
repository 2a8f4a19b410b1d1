"""Clipping in place refuses tensors that share an element, and takes those that only interleave: against sets of element numbers.

(What is refused launches nothing.)"""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2008_11343_b200 import binding as B
from paper_2008_11343_b200 import operators as O


def refused(ts):
    tl = O.TensorList(ts)
    try:
        tl.clip_grads(ts, 1.0)
    except B.ApmsError as e:
        assert "overlap in memory" in str(e)
        return True
    return False


def test_rows_that_meet_below_the_first():
    m = torch.ones(10, 16, device="cuda")
    for pair in ([m[:, :4], m[3]], [m[2:, :5], m[4:, 4:9]], [m[:6, 3:7], m[5:, :4]], [m[1::2, :4], m[2:, 3:6]], [m.view(-1)[40:50], m[:, 9:11]],
                 [m.view(5, 32)[:, :3], m[4:, :8]], [m[:, :8], m[:, 8:], m[7, 15:]]):
        assert refused(pair), [(t.shape, t.stride(), t.storage_offset()) for t in pair]
    assert (m == 1.0).all()
    for pair in ([m[:, :4], m[3, 4:]], [m[2:, :5], m[4:, 5:9]], [m[:5, 3:7], m[5:, :4]], [m[1::2, :4], m[::2, 3:6]], [m.view(-1)[43:50], m[:, 8:11]],
                 [m.view(5, 32)[:, :3], m[1::2, :8]], [m[:, :8], m[:, 8:]]):
        assert not refused(pair), [(t.shape, t.stride(), t.storage_offset()) for t in pair]


@pytest.mark.parametrize("seed", range(6))
def test_against_sets_of_elements(seed):
    rng = random.Random(seed)
    room = torch.ones(400, device="cuda", dtype=torch.bfloat16)
    index = torch.arange(400)
    found = {True: 0, False: 0}
    for _ in range(120):
        ts, sets = [], []
        for _ in range(rng.choice([2, 2, 3])):
            cols = rng.randint(1, 9)
            stride = rng.choice([16, 16, rng.randint(cols, 40)])
            rows, at = rng.randint(1, 8), rng.randint(0, 60)
            stride = max(stride, cols)
            args = ((rows, cols), (stride, 1), at)
            ts.append(room.as_strided(*args))
            sets.append(set(index.as_strided(*args).flatten().tolist()))
        want = sum(map(len, sets)) > len(set().union(*sets))
        assert refused(ts) == want, [(t.shape, t.stride(), t.storage_offset()) for t in ts]
        found[want] += 1
    assert min(found.values()) > 10
