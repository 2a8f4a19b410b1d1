"""Derivatives of derivatives: rms_norm has the first ones only and says so, with stand-ins for the two kernels (no GPU)."""
import os
import sys

import pytest
import torch

from paper_2008_11343_b200 import operators as O

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def forward(x, weight, residual=None, eps=1e-6):
    h = x.detach() if residual is None else x.detach() + residual.detach()
    rstd = (h.square().mean(-1) + eps).rsqrt()
    return h * rstd[..., None] * weight.detach(), x if residual is None else h, rstd


def backward(dy, h, weight, rstd, dh=None):
    dy, h, w, rstd = dy.detach(), h.detach(), weight.detach(), rstd[..., None]
    xh, a = h * rstd, w * dy
    dx = rstd * (a - xh * (a * xh).mean(-1, keepdim=True))
    return dx if dh is None else dx + dh.detach(), (dy * xh).flatten(0, -2).sum(0)


def plain(x, w, r):
    h = x if r is None else x + r
    return h * (h.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w, h


@pytest.fixture
def leaves(monkeypatch):
    monkeypatch.setattr(O, "rms_norm_forward", forward)
    monkeypatch.setattr(O, "rms_norm_backward", backward)
    gen = torch.Generator().manual_seed(1)
    return [torch.randn(*s, generator=gen, dtype=torch.float64).requires_grad_() for s in ((3, 5), (5,), (3, 5))]


@pytest.mark.parametrize("junction", [False, True])
@pytest.mark.parametrize("loss", [lambda y: y.square().sum(), lambda y: y.sum()], ids=["curved", "linear"])
def test_second_derivatives_are_refused_not_dropped(leaves, junction, loss):
    x, w, r = leaves
    out = O.rms_norm(x, w, r if junction else None)
    y = out[0] if junction else out
    inner = loss(y)
    grads = torch.autograd.grad(inner, [x, w], create_graph=True)
    want = torch.autograd.grad(loss(plain(x, w, r if junction else None)[0]), [x, w])
    assert all(torch.allclose(a, b, atol=1e-9) for a, b in zip(grads, want))          # the first ones are there
    with pytest.raises(RuntimeError, match="second derivative"):
        (inner + 10 * grads[1].square().sum() + x.sum() + w.sum()).backward()


def test_first_derivatives_and_the_stream_alone(leaves):
    x, w, r = leaves
    y, h = O.rms_norm(x, w, r)
    (y.square().sum() + h.sin().sum()).backward()
    want = torch.autograd.grad(sum(f(t) for f, t in zip((lambda t: t.square().sum(), lambda t: t.sin().sum()), plain(x, w, r))), [x, w, r])
    assert all(torch.allclose(t.grad, g, atol=1e-9) for t, g in zip((x, w, r), want)) and not x.grad.requires_grad
    _, h = O.rms_norm(x, w, r)
    dx, = torch.autograd.grad(h.square().sum(), x, create_graph=True)                 # the norm takes no part: h = x + r
    dxx, = torch.autograd.grad(dx.sum(), x)
    assert torch.allclose(dxx, torch.full_like(dxx, 2.0))


def test_the_example_refuses_them_too(monkeypatch):
    import train_block

    def eight_bit(x, weight, residual=None, eps=1e-6, group=0):
        y, h, rstd = forward(x, weight, residual, eps)
        return y, torch.ones(*y.shape[:-1], 1, dtype=y.dtype), h, rstd

    monkeypatch.setattr(O, "rms_norm_fp8", eight_bit)
    monkeypatch.setattr(O, "rms_norm_backward", lambda *a: (*backward(*a), backward(*a)[0]))
    x, w, r = (torch.randn(*s, dtype=torch.float64).requires_grad_() for s in ((3, 5), (5,), (3, 5)))
    y, h = train_block._EightBitNorm.apply(x, w, r)
    (y.sum() + h.sum()).backward(retain_graph=True)
    assert x.grad is not None and w.grad is not None
    with pytest.raises(RuntimeError, match="second derivative"):
        torch.autograd.grad(y.sum() + h.sum(), [x], create_graph=True)
