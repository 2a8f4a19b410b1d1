"""The gated linear recurrence where states are forgotten: what is gone leaves nothing in what is there, however large it was.

Bounds in units of 2^-24, step by step, of the magnitudes that are there (m_t = a_t m_(t-1) + z_t |x_t|), not of the largest in the channel."""
import pytest
import torch

import layers_oracle as oracle
from paper_2008_11343_b200 import operators as O

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
KINDS = [F32, BF16, F16]
U = oracle.U32
SPAN = 8                                                                            # steps from one kept state to the next


def normal(shape, kind=F32, scale=1.0, seed=0):
    return torch.empty(shape, device="cuda").normal_(0.0, scale, generator=torch.Generator(device="cuda").manual_seed(seed)).to(kind)


def uniform(shape, low, high, kind=F32, seed=0):
    return torch.empty(shape, device="cuda").uniform_(low, high, generator=torch.Generator(device="cuda").manual_seed(seed)).to(kind)


def taken(gate):
    """z, a and the units that a computed z = 1 / (1 + exp(gate)) is off by: of the exponential (binary32: the power of two 4, its argument's rest and the last rounding 2; 16 bits:
    the argument 1.5 |gate|, the power of two 4) only the share a, of the sum 1, of the reciprocal 2.  A gate of -infinity is exact."""
    g = gate.double()
    z, a = torch.sigmoid(-g), torch.sigmoid(g)
    exact = torch.isneginf(g)
    units = a * (6.0 if gate.dtype == F32 else 1.5 * g.abs().clamp(max=1e4) + 4) + 3
    return z, a, torch.where(exact, 0.0, units), exact


def scan(x, gate, state):
    """(h, its error, last, its error, and the states and errors before each step).  A step a h + z x with a = 1 - z: a is off by z's error and its own rounding, z x by z's error and its
    rounding, the sum by its rounding.  From span to span 20 roundings of m more: the product of 8 (or, joined for a segment, of two) factors 8, the sums that it or 1 minus it goes through 12."""
    z, a, units, exact = taken(gate)
    x = x.double()
    h = state.double()
    m, error = h.abs(), torch.zeros_like(h)
    hs, errors, before, errors_before = [], [], [], []
    for t in range(x.shape[1]):
        before.append(h)
        errors_before.append(error)
        zt, at, k, inexact = z[:, t], a[:, t], units[:, t], (~exact[:, t]).double()
        now = at * m + zt * x[:, t].abs()
        error = at * error + 1.01 * U * inexact * (m * (zt * k + at) + zt * x[:, t].abs() * (k + 1) + now)
        h, m = at * h + zt * x[:, t], now
        hs.append(h)
        errors.append(error)
        if (t + 1) % SPAN == 0:
            error = error + 20 * U * m
    joined = error if x.shape[1] % SPAN == 0 else error + 20 * U * m
    return torch.stack(hs, 1), torch.stack(errors, 1), h, joined, torch.stack(before, 1), torch.stack(errors_before, 1)


# One round; several of one sequence cut into segments; more slabs of channels than SMs, over several rounds; fewer, of two teams.
SHAPES = [(2, 40, 70), (2, 300, 71), (1, 1100, 24), (150, 200, 64), (40, 203, 130)]


def states(b, d, kind, size, seed):
    """No h of binary16 near its type's end."""
    return normal((b, d), scale=min(size, 1e4) if kind == F16 else size, seed=seed)


def check(x, gate, state):
    h, last, _ = O.gated_scan_forward(x, gate, state)
    want, error, want_last, last_error, _, _ = scan(x, gate, state)
    oracle.within(h, want, error, "h")
    oracle.within(last, want_last, last_error, "last")
    if x.dtype == F32:
        assert ((last - h[:, -1]).abs() <= error[:, -1] + last_error + 2 * U * want_last.abs()).all()
    return h, last


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("at", [0, 3, 7, 8, -1])
def test_minus_infinity_replaces_a_state_of_any_size(shape, kind, at):
    b, t, d = shape
    x, gate = normal(shape, kind, seed=1), uniform(shape, -1.0, 6.0, kind, seed=2)
    gate[:, at] = -float("inf")
    gate[:, t // 2] = -float("inf")
    h, last = check(x, gate, states(b, d, kind, 1e8, 3))
    assert torch.equal(h[:, at], x[:, at]) and torch.equal(h[:, t // 2], x[:, t // 2])
    if at == -1:
        assert torch.equal(last, x[:, -1].float())


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [1e4, 1e8])
def test_what_is_forgotten_soon_leaves_no_more_than_its_share(shape, kind, size):
    """z from 0.5 to 0.95."""
    b, t, d = shape
    check(normal(shape, kind, 1e-2, seed=4), uniform(shape, -3.0, 0.0, kind, seed=5), states(b, d, kind, size, 6))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SHAPES)
def test_an_outlier_among_small_values(shape, kind):
    """Held, forgotten and replaced states by turns."""
    b, t, d = shape
    x, gate = normal(shape, kind, 1e-2, seed=7), uniform(shape, -4.0, 8.0, kind, seed=8)
    x[:, 5], x[:, t // 2] = 3e4, -3e4
    gate[:, 20:30] = float("inf")
    check(x, gate, states(b, d, kind, 1e6, 9))


def gradient(dh, x, gate, state, dlast):
    """((dx, error), (dgate, error), (dstate, error)).  G = dh + k rounds once; k = G - z G is off by z's error and two roundings of G, from span to span by 20 of itself; a z = e z z by
    three errors of the exponential, two of z beside that and two roundings; h - x by the error of h and a rounding."""
    z, a, units, exact = taken(gate)
    _, _, _, _, before, before_error = scan(x, gate, state)
    exponential = 6.0 if gate.dtype == F32 else 1.5 * gate.double().abs().clamp(max=1e4) + 4
    x, dh = x.double(), dh.double()
    az = a * z
    k = dlast.double()
    size, error = k.abs(), torch.zeros_like(k)
    out = [[], [], [], []]
    for t in reversed(range(x.shape[1])):
        g, size = dh[:, t] + k, dh[:, t].abs() + size
        error = error + U * size
        zt, at, e = z[:, t], a[:, t], before[:, t] - x[:, t]
        dgate = g * e * az[:, t]
        relative = 3 * (exponential if gate.dtype == F32 else exponential[:, t]) + 8 + 3
        for values, v in zip(out, (zt * g, 1.01 * zt * (error + size * (units[:, t] + 1) * U), dgate,
                                   1.01 * (az[:, t] * (error * e.abs() + size * (before_error[:, t] + e.abs() * U)) + dgate.abs() * relative * U))):
            values.append(v)
        k, error, size = at * g, at * error + 1.01 * U * (~exact[:, t]).double() * size * (zt * units[:, t] + 2), at * size
        if t % SPAN == 0:
            error = error + 20 * U * size
    dx, dx_error, dg, dg_error = (torch.stack(v[::-1], 1) for v in out)
    return (dx, dx_error), (dg, dg_error), (k, error)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("low,high,at", [(-1.0, 6.0, 0), (-1.0, 6.0, 3), (-1.0, 6.0, 8), (-1.0, 6.0, -1), (-3.0, 0.0, None)])
def test_gradients_behind_a_state_that_is_gone(shape, kind, low, high, at):
    """The states that dgate takes are formed again, from the kept ones that may be as large as they like."""
    b, t, d = shape
    x, gate, state, dh, dlast = normal(shape, kind, seed=10), uniform(shape, low, high, kind, seed=11), states(b, d, kind, 1e8, 12), normal(shape, kind, 1e-2, seed=13), normal((b, d), F32, 1e-2, seed=14)
    if at is not None:
        gate[:, at] = gate[:, t // 2] = -float("inf")
    starts = O.gated_scan_forward(x, gate, state, keep=True)[2]
    for got, (want, error), name in zip(O.gated_scan_backward(dh, x, gate, starts, dlast), gradient(dh, x, gate, state, dlast), ("dx", "dgate", "dstate")):
        oracle.within(got, want, error, name)


@pytest.mark.parametrize("shape", [(3, 64), (5, 1001), (64, 1000)])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [1.0, 1e4, 1e8])
def test_one_token_replaces_a_state_of_any_size(shape, kind, size):
    """As a sequence of one step does; its sum h + z (x - h), where z is 1/2 or less, rounds x - h beside: z u |x - h|, within a u |h| + z u |x|."""
    b, d = shape
    x, gate, state = normal(shape, kind, 1e-2, seed=15), uniform(shape, -3.0, 6.0, kind, seed=16), states(b, d, kind, size, 17)
    gate[:, ::3] = -float("inf")
    want, error, _, _, _, _ = scan(x[:, None], gate[:, None], state)
    out = torch.empty_like(state)
    h = O.gated_scan_step(x, gate, state, out=out)
    oracle.within(h, want[:, 0], error[:, 0])
    oracle.within(out, want[:, 0], error[:, 0])
    assert torch.equal(h[:, ::3], x[:, ::3]) and torch.equal(out[:, ::3], x[:, ::3].float())
