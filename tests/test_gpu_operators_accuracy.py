"""8-bit output is the nearest there is, calls repeat themselves, and the backward pass of wide rows off the 16-byte boundary.

The number that is rounded to e4m3 is h rstd w (448 / a): both products, the quotient, the last product, a's own rounding and the one of
max |h w| times rstd, 6u of it (u = 2^-24), and h's; rstd itself cancels.  Within 8u of a tie either neighbour is right, elsewhere only the
nearest is."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2008_11343_b200 import operators as O
from test_gpu_operators import BF16, EPS, F16, F32, U, activation, check_backward, check_fp8, weight_of


def check_nearest_e4m3(q, ratio, slack):
    """q is the e4m3 value nearest to `ratio` (binary64), or its neighbour where the tie between them is within `slack`."""
    size = ratio.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(size.clamp(min=2.0 ** -6))) - 3)
    low = torch.floor(size / step) * step
    below, above = (size - low - step / 2 <= slack), (size - low - step / 2 >= -slack)
    got = q.double().abs()
    right = ((got == low) & below) | ((got == low + step) & above)
    assert right.all(), f"{int((~right).sum())} of {q.numel()}: {got[~right][:3]} for {ratio[~right][:3]}"
    assert ((q.double() == 0) | (torch.sign(q.double()) == torch.sign(ratio))).all()


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("kind", [(BF16, BF16, BF16), (BF16, None, BF16), (F16, F16, F16), (F32, F32, F32), (BF16, F32, F32)], ids=str)
@pytest.mark.parametrize("rows,width", [(2048, 4096), (333, 1000), (97, 1003), (5000, 128)])
def test_eight_bit_values_are_the_nearest(rows, width, kind, group):
    """bfloat16 products often lie exactly between two e4m3 values; there, and only there, may a rounding of the scale decide."""
    dt, rt, wt = kind
    x = activation(rows, width, dt, 1)
    r = None if rt is None else activation(rows, width, rt, 2, scale=2.0)
    w = weight_of(width, wt, 3)
    got = O.rms_norm_fp8(x, w, r, eps=EPS, group=group)
    check_fp8(x, w, r, group, got)
    h = x.double() if r is None else x.double() + r.double()
    hw, size = h * w.double(), group or width                                # rstd cancels between y and its scale
    a = torch.cat([p.abs().amax(-1, keepdim=True).expand_as(p) for p in hw.split(size, -1)], -1)
    lost = (x.double().abs() + (0 if r is None else r.double().abs())) * U if r is not None else 0.0
    ratio = hw / a * 448.0
    check_nearest_e4m3(got[0], ratio, 8 * U * ratio.abs() + lost * w.double().abs() / a * 448.0)


@pytest.mark.parametrize("group", [None, 0, 128])
def test_the_same_call_gives_the_same_bits(group):
    for width in (64, 1000, 1001, 4096, 70_000):
        x, r, w = activation(301, width, BF16, 4), activation(301, width, BF16, 5), weight_of(width, BF16, 6)
        call = (lambda: O.rms_norm_forward(x, w, r)) if group is None else (lambda: O.rms_norm_fp8(x, w, r, group=group))
        first = call()
        for _ in range(3):
            for a, b in zip(first, call()):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("kind", [(F32, F32, F32), (BF16, BF16, BF16), (BF16, F32, F32), (F16, F16, F32), (F16, F32, F16), (BF16, BF16, F32)], ids=str)
@pytest.mark.parametrize("width", [4099, 6251, 8191, 12_001])
@pytest.mark.parametrize("carried", [False, True])
def test_gradients_of_wide_rows_off_the_boundary(kind, width, carried):
    dt, ht, wt = kind
    rows = 613                                                               # several rows a CTA
    dy = activation(rows, width, dt, 9, scale=0.1)
    h = activation(rows, width, ht, 10, scale=2.0)
    dh = activation(rows, width, ht, 11, scale=0.1) if carried else None
    w = weight_of(width, wt, 12)
    rstd = (1.0 / (h.double().square().mean(-1) + EPS).sqrt()).float()
    check_backward(dy, h, w, rstd, dh, O.rms_norm_backward(dy, h, w, rstd, dh))
