"""rstd and the backward pass's mean, of rows of one value and of rows wider than a CTA holds.

Tolerances, from the roundings that the kernels make (u = 2^-24):

  rstd       h rounded once (u in each, so 2u in a square); a chain of at most 64 additions in a lane, one more, 5 in a warp, 15 over the
             warps: 85u; 1 / width, the product with it, eps: 3u.  90u under the root: 45u.  The reciprocal root: 2 units in the last place, 4u.  Below 50u.
  mean       xh, a and their product are rounded once each, the mean twice, whatever the width.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2008_11343_b200 import operators as O
from test_gpu_operators import BF16, EPS, F32, ROUND, U, activation, forward64, near, weight_of

RSTD = 50 * U

WIDE = [128, 1000, 4096, 16_383, 16_384, 32_768, 50_001, 65_544, 1 << 18, 1 << 20]


@pytest.mark.parametrize("width", WIDE + [1 << 24])
@pytest.mark.parametrize("dt,rt", [(F32, None), (F32, F32), (BF16, None), (BF16, BF16), (BF16, F32)], ids=str)
def test_rstd_of_equal_and_of_random_elements(dt, rt, width):
    """Rows of one value are the hard ones: each addition of a chain rounds the same way."""
    rows = 2 if width > 1 << 20 else 7
    w = weight_of(width, dt, 7)
    values = torch.tensor([1.1, 0.3, 3.7e-3, 1e4, 0.7, 1.9, 5.3][:rows], device="cuda")
    for x in (values[:, None].expand(rows, width).to(dt).contiguous(), activation(rows, width, dt, 8)):
        r = None if rt is None else (values.flip(0)[:, None] * 0.37).expand(rows, width).to(rt).contiguous()
        y, _, rstd = O.rms_norm_forward(x, w, r, eps=EPS)
        _, want, y64 = forward64(x, w, r)
        near(rstd, want, want * RSTD, "rstd")
        rel, least = ROUND[dt]
        lost = 0 if r is None else (x.double().abs() + r.double().abs()) * U * want[:, None] * w.double().abs()
        near(y, y64, y64.abs() * (RSTD + 4 * U + rel) + lost + least, "y")
        _, scales, _, rstd8 = O.rms_norm_fp8(x, w, r, eps=EPS)
        near(rstd8, want, want * RSTD, "rstd")
        near(scales[:, 0], y64.abs().amax(1) / 448.0, y64.abs().amax(1) / 448.0 * (RSTD + 6 * U) + (0 if r is None else lost.amax(1) / 448.0), "scales")


@pytest.mark.parametrize("width", [65_544, 1 << 18, 1 << 20])
@pytest.mark.parametrize("dt,ht", [(F32, F32), (BF16, BF16), (BF16, F32)], ids=str)
def test_the_mean_of_a_wide_row_in_the_backward_pass(dt, ht, width):
    """Equal elements: dx is the small difference of a and xh mean(a xh), so an error of the mean shows whole."""
    rows = 3
    h = torch.tensor([1.1, 0.3, 3.7], device="cuda")[:, None].expand(rows, width).to(ht).contiguous()
    dy = torch.tensor([0.7, 1.9, 0.013], device="cuda")[:, None].expand(rows, width).to(dt).contiguous()
    w = torch.full((width,), 1.3, device="cuda").to(dt)
    rstd = (1.0 / (h.double().square().mean(-1) + EPS).sqrt()).float()
    dx, dw, *_ = O.rms_norm_backward(dy, h, w, rstd)
    xh, a = h.double() * rstd.double()[:, None], w.double() * dy.double()
    mean = (a * xh).mean(-1, keepdim=True)
    want = rstd.double()[:, None] * (a - xh * mean)
    rel, least = ROUND[dt]
    terms = rstd.double()[:, None] * (a.abs() + xh.abs() * mean.abs())
    near(dx, want, terms * 8 * U + want.abs() * rel + least, "dx")
    near(dw, (dy.double() * xh).sum(0), (dy.double() * xh).abs().sum(0) * (rel + 8 * U), "dweight")
