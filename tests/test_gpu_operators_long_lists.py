"""Lists of more than 8192 tiles (32 KB each): their sums go over groups of tiles, several CTAs and a ticket.

Tolerances: squares are summed in binary64 (binary32 ones are exact there), the root is rounded once: u = 2^-24.  A clipped element has the
factor's rounding, the product's and the output type's."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2008_11343_b200 import operators as O
from test_gpu_operators import BF16, F16, F32, ROUND, U, gen, near

ONCE = U * (1 + 2.0 ** -10)

LISTS = {
    "8300 of one element": ([1] * 8300, [BF16]),
    "one of 8200 tiles": ([8200 * 8192 - 5], [F32]),                         # nine groups of one tensor
    "long ones among short": ([5, 1030 * 16384 + 77, 3] + [9000] * 3500 + [1024 * 16384, 1] + [20_001] * 20, [BF16, BF16, F32]),
}


def tensors_of(name):
    sizes, types = LISTS[name]
    g = gen(21)
    return [torch.empty(n, dtype=types[k % len(types)], device="cuda").normal_(0.0, 10.0 ** (-(k % 4)), generator=g) for k, n in enumerate(sizes)]


@pytest.mark.parametrize("name", LISTS)
def test_norm_and_clipping_of_a_long_list(name):
    ts = tensors_of(name)
    tl = O.TensorList(ts)
    squares = torch.stack([t.double().square().sum() for t in ts])
    want, wants = squares.sum().sqrt(), squares.sqrt()
    norm, norms = tl.grad_norm(ts)
    near(norm, want, want * ONCE)
    near(norms, wants, wants * ONCE)
    limit = 0.37
    c = limit / float(want)
    flat = torch.empty(tl.numel, device="cuda")
    before = torch.cat([t.float() for t in ts])
    for _ in range(3):                                                       # the ticket is back at zero after each call
        flat.fill_(7.0)
        assert torch.equal(tl.clip_grads(ts, limit, out=flat), norm)
        near(flat, before.double() * c, (before.double() * c).abs() * 3 * ONCE + 2.0 ** -150)
        again, agains = tl.grad_norm(ts)
        assert torch.equal(again, norm) and torch.equal(agains, norms)
    assert torch.equal(torch.cat([t.float() for t in ts]), before)
    assert torch.equal(tl.clip_grads(ts, limit), norm)                       # in place
    at = 0
    for t in ts:
        wanted = before[at:at + t.numel()].double() * c
        at += t.numel()
        rel, least = ROUND[t.dtype]
        near(t, wanted, wanted.abs() * (2 * ONCE + rel) + least)


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("sizes", [[3], [100_003, 7], [9000] * 300], ids=lambda s: f"{len(s)}x{s[0]}")
def test_the_norm_is_rounded_once(sizes, dtype):
    ts = [torch.empty(n, dtype=dtype, device="cuda").normal_(generator=gen(22 + k)) for k, n in enumerate(sizes)]
    norm, norms = O.TensorList(ts).grad_norm(ts)
    squares = torch.stack([t.double().square().sum() for t in ts])
    near(norm, squares.sum().sqrt(), squares.sum().sqrt() * ONCE)
    near(norms, squares.sqrt(), squares.sqrt() * ONCE)
