"""Dense gradients whose elements lie in another order than their indexes': transposed, channels last.

The norm and clipping in place take them as the run of memory that they are; the flat gradient has the elements in the order of their
indexes.  Tolerances: u = 2^-24 for the norm's root, 2u and the output type's rounding for a clipped element."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2008_11343_b200 import binding as B
from paper_2008_11343_b200 import operators as O
from test_gpu_operators import BF16, F16, F32, ROUND, U, gen, near

ONCE = U * (1 + 2.0 ** -10)


def gradients(dtype):
    g = gen(31)

    def normal(*shape):
        return torch.empty(*shape, dtype=dtype, device="cuda").normal_(generator=g)

    return [normal(301, 77).t(), normal(9000), normal(6, 33, 5, 7).contiguous(memory_format=torch.channels_last), normal(5, 4, 3).permute(2, 0, 1),
            normal(1, 130).t(), normal(40, 50)[:, 7:20], normal(129, 257).t()]


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
def test_dense_gradients_in_any_order(dtype):
    ts = gradients(dtype)
    before = [t.clone() for t in ts]                                         # keeps the strides
    assert not ts[0].is_contiguous() and not ts[2].is_contiguous()
    tl = O.TensorList(ts)
    squares = torch.stack([t.double().square().sum() for t in ts])
    want, wants = squares.sum().sqrt(), squares.sqrt()
    norm, norms = tl.grad_norm(ts)
    near(norm, want, want * ONCE)
    near(norms, wants, wants * ONCE)
    c, (rel, least) = 2.0 / float(want), ROUND[dtype]
    for out in (F32, dtype):
        flat = torch.full((tl.numel + 8,), 7.0, dtype=out, device="cuda")
        assert torch.equal(tl.clip_grads(ts, 2.0, out=flat[:-8]), norm) and (flat[-8:] == 7.0).all()
        wanted = torch.cat([t.double().flatten() for t in before]) * c       # by index
        near(flat[:-8], wanted, wanted.abs() * (2 * ONCE + ROUND[out][0]) + ROUND[out][1])
    assert all(torch.equal(a, b) for a, b in zip(ts, before))
    assert torch.equal(tl.clip_grads(ts, 2.0), norm)
    for t, b in zip(ts, before):
        wanted = b.double() * c
        near(t, wanted, wanted.abs() * (2 * ONCE + rel) + least)


def test_the_order_belongs_to_the_list():
    a = torch.ones(4, 6, device="cuda")
    tl = O.TensorList([a.t()])
    with pytest.raises(ValueError, match="strides"):
        tl.grad_norm([torch.ones(6, 4, device="cuda")])
    with pytest.raises(ValueError, match="strides"):
        O.TensorList([torch.ones(6, 4, device="cuda")]).grad_norm([a.t()])
    for bad in (torch.ones(8, 12, device="cuda")[::2, ::2].t(), torch.ones(1, 4, device="cuda").expand(3, 4)):
        with pytest.raises(ValueError, match="rows of consecutive"):
            O.TensorList([bad])


def test_a_flat_gradient_in_the_memory_of_a_tensor_in_another_order():
    flat = torch.ones(24, device="cuda")
    turned = [flat.view(4, 6).t()]
    with pytest.raises(B.ApmsError, match="overlaps the flat gradient"):
        O.TensorList(turned).clip_grads(turned, 1.0, out=flat)
    assert (flat == 1.0).all()
