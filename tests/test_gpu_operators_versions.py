"""What clip_grads writes, autograd knows of: a tensor that a graph has saved and that is then clipped raises in the graph's backward pass."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2008_11343_b200 import operators as O


def saved(n=100):
    t = torch.full((n,), 3.0, device="cuda")
    x = torch.ones(n, device="cuda", requires_grad=True)
    return t, x, (x * t).sum()                                               # keeps t for x's gradient


def test_clipping_in_place_is_seen():
    t, x, loss = saved()
    other = torch.ones(5, device="cuda")
    O.TensorList([other, t]).clip_grads((v for v in (other, t)), 1.0)       # any iterable
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_the_flat_gradient_is_seen():
    t, x, loss = saved()
    grads = [torch.ones(60, device="cuda"), torch.ones(40, device="cuda")]
    O.TensorList(grads).clip_grads(grads, 1.0, out=t)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_a_view_of_what_is_written_is_seen():
    t, x, loss = saved()
    half = [t[:50]]
    O.TensorList(half).clip_grads(half, 1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_what_is_only_read_or_refused_stays_as_it_was():
    t, x, loss = saved()
    tl, flat = O.TensorList([t]), torch.empty(100, device="cuda")
    tl.grad_norm([t])
    tl.clip_grads([t], 1.0, out=flat)
    with pytest.raises(Exception, match="max_norm"):
        tl.clip_grads([t], -1.0)
    loss.backward()
    assert (x.grad == 3.0).all()


def test_tensors_without_a_version():
    with torch.inference_mode():
        t = torch.full((100,), 3.0, device="cuda")
    tl = O.TensorList([t])
    assert float(tl.clip_grads([t], 15.0)) == 30.0
    assert (t == 1.5).all()
