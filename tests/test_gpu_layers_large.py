"""The layers' operators where places pass 2^31 and 2^32 elements, by the parts that lie behind them."""
import numpy as np
import pytest
import torch

import layers_oracle as oracle
from paper_2008_11343_b200 import operators as O

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def freed():
    yield
    torch.cuda.empty_cache()


def normal(shape, seed, scale=1.0):
    return torch.empty(shape, dtype=BF16, device="cuda").normal_(0.0, scale, generator=torch.Generator(device="cuda").manual_seed(seed))


@pytest.mark.parametrize("width", [65536, 65535])
def test_rows_of_a_large_table(width):
    """4.6 G elements."""
    vocabulary = 70_000
    weight = normal((vocabulary, width), 1)
    tokens = torch.tensor([69_999, 3, 35_000, 69_998, 69_999], device="cuda")
    oracle.within(O.embedding_forward(tokens, weight, 3.0), *oracle.embedding(torch.arange(4, device="cuda")[[3, 0, 1, 2, 3]], weight[[3, 35_000, 69_998, 69_999]], 3.0))
    del weight
    for count in (5, 1100):
        many = tokens.repeat(count // 5)
        dout = normal((count, width), 2)
        got = O.embedding_backward(dout, many, vocabulary)
        want, error = oracle.embedding_gradient(dout, torch.tensor([3, 0, 1, 2, 3], device="cuda").repeat(count // 5), 4, 1.0)
        rows = [3, 35_000, 69_998, 69_999]
        oracle.within(got[rows], want, error)
        got[rows] = 0
        assert not got.any()
        del got


@pytest.mark.parametrize("width", [4104, 4103])
def test_a_large_mask(width):
    """4.3 G elements; the last rows' blocks are those of their elements' indexes."""
    rows = (1 << 20) + 3
    x = normal((rows, width), 3)
    h, used = O.dropout_forward(x, 0.3, torch.tensor([5, 6], device="cuda"), 7)
    for row in (0, 1 << 19, rows - 1):
        first = row * width
        blocks = np.arange(first // 8, (first + width + 7) // 8)
        words = oracle.philox([blocks, np.full(len(blocks), 7), np.full(len(blocks), 6), np.zeros(len(blocks))], [5, 0], 7)
        bits = np.stack([half for w in words for half in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=1).ravel()[first % 8:first % 8 + width]
        border = int(np.floor(65536 * 0.3 + 0.5))
        want = torch.where(torch.from_numpy(bits >= border).cuda(), x[row].double() * (65536 / (65536 - border)), 0.0)
        oracle.within(h[row], want, want.abs() * 2.01 * oracle.U32)


def test_many_sequences():
    """2.5 G elements a tensor."""
    shape = (600, 100, 40_960)
    x, gate, dh = normal(shape, 4), normal(shape, 5, 2.0), normal(shape, 6)
    h, last, starts = O.gated_scan_forward(x, gate, None, keep=True)
    dx, dgate, dstate = O.gated_scan_backward(dh, x, gate, starts)
    for part in (slice(0, 1), slice(599, 600)):
        one = [t[part, :, -300:] for t in (x, gate, dh)]
        want, error, want_last, last_error, _ = oracle.scan(one[0], one[1])
        oracle.within(h[part, :, -300:], want, error)
        oracle.within(last[part, -300:], want_last, last_error)
        for got, (value, off) in zip((dx[part, :, -300:], dgate[part, :, -300:], dstate[part, -300:]), oracle.scan_gradient(one[2], one[0], one[1])):
            oracle.within(got, value, off)
