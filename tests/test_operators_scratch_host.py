"""Scratch memory of a list of tensors: its size, and what is refused before anything is enqueued (no GPU)."""
import pytest

from paper_2008_11343_b200 import binding as B
from paper_2008_11343_b200 import build as libbuild


@pytest.fixture(scope="module", autouse=True)
def lib():
    libbuild.build()
    return B.load()


def test_scratch_is_what_the_calls_write():
    for sizes in ([8], [8, 0, 100_000], [1] * 9000):
        h = B.apms_tensors_create(sizes, [B.GRAD_F32] * len(sizes))
        scratch, whole = B.apms_tensors_scratch_bytes(h), B.apms_tensors_workspace_bytes(h)
        assert scratch % 256 == 0 and 8 * len([n for n in sizes if n]) < scratch < whole           # a double a tile, the ticket
        B.apms_tensors_destroy(h)
    assert B.apms_tensors_scratch_bytes(None) == 0


def test_scratch_is_refused_without_a_workspace():
    h = B.apms_tensors_create([8], [B.GRAD_F32])
    for list_, p in ((h, 256), (h, None), (None, 256)):
        with pytest.raises(B.ApmsError, match="no workspace") as e:
            B.apms_tensors_use_scratch(list_, p, 1 << 20, None)
        assert e.value.status == B.ERR_BAD_STATE
    B.apms_tensors_destroy(h)
