"""The embedding and its gradient, dropout, and the gated linear recurrence against plain 64-bit forms: odd sizes, types, strides and addresses, values that are not finite."""
import pytest
import torch

import layers_oracle as oracle
from paper_2008_11343_b200 import binding as B
from paper_2008_11343_b200 import operators as O

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
KINDS = [F32, BF16, F16]


def gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(shape, kind=F32, scale=1.0, seed=0, pad=0, offset=0):
    """Rows `pad` elements further apart, the first of them `offset` elements into its buffer."""
    rows = 1
    for s in shape[:-1]:
        rows *= s
    flat = torch.empty(rows * (shape[-1] + pad) + offset, device="cuda").normal_(0.0, scale, generator=gen(seed)).to(kind)
    return flat[offset:].view(*shape[:-1], shape[-1] + pad)[..., :shape[-1]]


# ------------------------------------------------------------------------------------------ embedding

def tokens_for(count, vocabulary, seed, kind=torch.int64, hot=0.3):
    """Some tokens often, some outside the vocabulary."""
    t = torch.randint(0, vocabulary, (count,), device="cuda", generator=gen(seed))
    u = torch.rand(count, device="cuda", generator=gen(seed + 1))
    t[u < hot] = vocabulary // 2
    t[u > 0.95] = torch.tensor([-1, -100, vocabulary, 2 ** 31 - 1], device="cuda")[torch.randint(0, 4, (int((u > 0.95).sum()),), device="cuda", generator=gen(seed))]
    return t.to(kind)


EMBEDDINGS = [(1, 1, 1), (1, 30522, 64), (3, 7, 8), (31, 2, 65), (257, 300, 1000), (1000, 33, 1001), (4097, 70001, 24), (513, 255, 1032), (2048, 256, 136), (700, 65536, 4), (130, 40, 3333), (1024, 30, 72), (1025, 30, 72), (1100, 2000, 2600), (3000, 5000, 200), (2000, 9000, 1001), (1500, 200000, 8)]


@pytest.mark.parametrize("count,vocabulary,width", EMBEDDINGS)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("out", KINDS)
def test_lookup(count, vocabulary, width, kind, out):
    tokens, weight = tokens_for(count, vocabulary, 1), normal((vocabulary, width), kind, seed=2)
    within = oracle.embedding(tokens, weight, 7.3)
    oracle.within(O.embedding_forward(tokens, weight, 7.3, dtype=out), *within)


@pytest.mark.parametrize("count,vocabulary,width", EMBEDDINGS)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("out", KINDS)
def test_gradient(count, vocabulary, width, kind, out):
    tokens, dout = tokens_for(count, vocabulary, 3, torch.int32), normal((count, width), kind, seed=4)
    got = O.embedding_backward(dout, tokens, vocabulary, 0.7, dtype=out)
    oracle.within(got, *oracle.embedding_gradient(dout, tokens, vocabulary, 0.7))


@pytest.mark.parametrize("hot", [0.0, 1.0])
@pytest.mark.parametrize("count,vocabulary,width", [(20_000, 30522, 40), (70_001, 1 << 18, 8), (33_000, 5, 1032), (9000, 1 << 24, 1)])
def test_gradient_of_many_tokens(count, vocabulary, width, hot):
    """More than one group of runs, two to four passes of the sort; one token everywhere (hot = 1) or all alike."""
    tokens, dout = tokens_for(count, vocabulary, 5, hot=hot), normal((count, width), BF16, seed=6)
    got = O.embedding_backward(dout, tokens, vocabulary, dtype=F32)
    oracle.within(got, *oracle.embedding_gradient(dout, tokens, vocabulary, 1.0))
    assert torch.equal(got, O.embedding_backward(dout, tokens, vocabulary, dtype=F32))              # the same bits again


def test_no_token_lies_in_the_vocabulary():
    tokens = torch.full((77,), -100, device="cuda")
    assert not O.embedding_forward(tokens, normal((9, 16)), 1.0).any()
    assert not O.embedding_backward(normal((77, 16)), tokens, 9).any()
    nothing = tokens[:0]
    assert O.embedding_forward(nothing, normal((9, 16))).shape == (0, 16)
    assert not O.embedding_backward(normal((0, 16)), nothing, 9).any()


def test_values_that_are_not_finite_stay_in_their_rows():
    tokens = torch.tensor([3, 1, 3, 8, 1, -1], device="cuda")
    dout = normal((6, 40), F32, seed=7)
    dout[0, 3], dout[3, 5], dout[5, 7] = float("inf"), float("nan"), float("nan")          # the last one's token has no row
    got = O.embedding_backward(dout, tokens, 10)
    want = torch.zeros(10, 40, dtype=torch.float64, device="cuda").index_add_(0, tokens[:5], dout[:5].double())
    oracle.within(got, want, want.abs() * 4 * oracle.U32 + 1e-6)
    weight = normal((10, 40))
    weight[2] = float("nan")
    assert torch.isfinite(O.embedding_forward(tokens, weight, 2.0)).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("width,pad,offset", [(64, 8, 0), (64, 3, 0), (64, 0, 1), (50, 6, 2), (33, 7, 8), (50, 0, 1), (550, 2, 0), (2, 0, 0)])
def test_rows_anywhere(kind, width, pad, offset):
    tokens = tokens_for(500, 90, 8).view(20, 25)
    weight = normal((90, width), kind, seed=9, pad=pad, offset=offset)
    got = O.embedding_forward(tokens.t(), weight, 1.5)
    oracle.within(got, *oracle.embedding(tokens.t(), weight, 1.5))
    dout = normal((500, width), kind, seed=10, pad=pad, offset=offset)
    flat = torch.full((90 * width + 2 * offset + 64,), 7.0, dtype=kind, device="cuda")
    place = flat[offset:offset + 90 * width].view(90, width)
    assert O.embedding_backward(dout.view(20, 25, width) if pad == 0 else dout, tokens if pad == 0 else tokens.flatten(), 90, out=place) is not None
    oracle.within(place, *oracle.embedding_gradient(dout, tokens, 90, 1.0))
    assert (flat[:offset] == 7).all() and (flat[offset + 90 * width:] == 7).all()


def test_lookup_is_differentiable_into_its_weight():
    weight = normal((50, 24), BF16, seed=11).requires_grad_()
    tokens = tokens_for(300, 50, 12).view(3, 100)
    out = O.embedding(tokens, weight, 4.0, dtype=F32)
    dout = normal((3, 100, 24), F32, seed=13)
    out.backward(dout)
    assert weight.grad.dtype == BF16
    oracle.within(weight.grad, *oracle.embedding_gradient(dout, tokens, 50, 4.0))


# ------------------------------------------------------------------------------------------ dropout

def rng_of(seed, step):
    return torch.tensor([seed, step], device="cuda")


@pytest.mark.parametrize("shape", [(1, 1), (1, 8), (3, 5), (7, 64), (5, 1001), (33, 257), (2, 3, 1032), (1000, 8), (123, 1), (640, 4096)])
@pytest.mark.parametrize("kind,stream", [(F32, None), (BF16, None), (F16, None), (F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
def test_dropout(shape, kind, stream):
    x = normal(shape, kind, seed=20)
    residual = None if stream is None else normal(shape, stream, 2.0, seed=21)
    seed, step = -(2 ** 62) + 12345, (7 << 32) + 99
    h, used = O.dropout_forward(x, 0.3, rng_of(seed, step), 2 ** 32 - 1, residual)
    assert h.dtype == (stream or kind) and used.tolist() == [seed, step]
    oracle.within(h, *oracle.dropout(x, 0.3, seed, step, 2 ** 32 - 1, residual))
    dh = normal(shape, stream or kind, seed=22)
    dx = O.dropout_backward(dh, 0.3, used, 2 ** 32 - 1, dtype=kind)
    assert dx.dtype == kind
    oracle.within(dx, *oracle.dropout(dh, 0.3, seed, step, 2 ** 32 - 1))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("width,pad,offset", [(64, 8, 0), (64, 8, 8), (64, 0, 1), (64, 3, 0), (1001, 0, 0), (1001, 23, 0), (4, 4, 0), (24, 8, 0)])
def test_dropout_of_rows_anywhere(kind, width, pad, offset):
    x, r = normal((37, width), kind, seed=23, pad=pad, offset=offset), normal((37, width), kind, seed=24)
    h, _ = O.dropout_forward(x, 0.25, rng_of(5, 6), 1, r)
    oracle.within(h, *oracle.dropout(x, 0.25, 5, 6, 1, r))
    h, _ = O.dropout_forward(r, 0.25, rng_of(5, 6), 1, x)
    oracle.within(h, *oracle.dropout(r, 0.25, 5, 6, 1, x))


@pytest.mark.parametrize("p", [0.0, 1.0, 2.0 ** -18, 1 - 2.0 ** -18, 2.0 ** -16, 0.5])
def test_dropout_at_the_ends(p):
    x, r = normal((33, 100), BF16, seed=25), normal((33, 100), F32, seed=26)
    x[3, 3], x[4, 4], x[5, 5] = float("inf"), float("nan"), -float("inf")
    h, used = O.dropout_forward(x, p, rng_of(1, 2), 3, r)
    oracle.within(h, *oracle.dropout(x, p, 1, 2, 3, r))
    if p == 0.0:
        assert torch.equal(h.nan_to_num(), (x.float() + r).nan_to_num())
    if round(p * 65536) == 65536:
        assert torch.equal(h, r)                                                    # what is dropped counts as 0 whatever it is


def test_masks_differ_by_seed_step_and_site_and_keep_their_share():
    x = torch.ones(1 << 20, device="cuda")
    masks = [O.dropout_forward(x, 0.1, rng_of(*k), site)[0] > 0 for *k, site in [(1, 0, 0), (2, 0, 0), (1, 1, 0), (1, 0, 1), (1, 1 << 32, 0), (1 + (1 << 32), 0, 0)]]
    n = x.numel()
    for m in masks:                                                                 # 5.5 standard deviations of a share of 0.9
        assert abs(float(m.sum()) - 0.9 * n) < 5.5 * (0.09 * n) ** 0.5 + n * 2.0 ** -17
    for i in range(len(masks)):
        for j in range(i):                                                          # and of the share of 0.82 that is the same in two of them
            assert abs(float((masks[i] == masks[j]).sum()) - 0.82 * n) < 5.5 * (0.1476 * n) ** 0.5 + n * 2.0 ** -15


def test_dropout_is_differentiable_whatever_happens_to_the_numbers():
    x, r, rng = normal((20, 33), BF16, seed=27).requires_grad_(), normal((20, 33), F32, seed=28).requires_grad_(), rng_of(8, 9)
    h = O.dropout(x, 0.4, rng, 5, r)
    rng[1] += 1                                                                     # the next step's, before the backward pass
    dh = normal((20, 33), F32, seed=29)
    h.backward(dh)
    assert torch.equal(r.grad, dh) and x.grad.dtype == BF16
    oracle.within(x.grad, *oracle.dropout(dh, 0.4, 8, 9, 5))
    assert O.dropout_forward(normal((0, 8)), 0.4, rng, 5)[1].tolist() == [8, 10]


# ------------------------------------------------------------------------------------------ gated linear recurrence

SCANS = [(1, 1, 1), (2, 16, 64), (3, 17, 65), (1, 129, 1001), (5, 33, 8), (2, 300, 72), (40, 7, 96), (1, 515, 64), (3, 250, 130), (9, 20, 500), (2, 64, 1), (1, 40, 2050)]


def gates(shape, kind, seed, **more):
    return (normal(shape, kind, 1.5, seed=seed, **more) + torch.linspace(-1.0, 6.0, shape[-1], device="cuda").to(kind)).clamp(-16, 16)


def check_scan(x, gate, state, dh=None, dlast=None):
    h, last, starts = O.gated_scan_forward(x, gate, state, keep=True)
    want, error, want_last, last_error, _ = oracle.scan(x, gate, state)
    oracle.within(h, want, error, "h")
    oracle.within(last, want_last, last_error, "last")
    again, last_again, none = O.gated_scan_forward(x, gate, state)
    assert none is None and torch.equal(again, h) and torch.equal(last, last_again)
    if dh is None:
        return
    grads = O.gated_scan_backward(dh, x, gate, starts, dlast)
    for got, (value, off), name in zip(grads, oracle.scan_gradient(dh, x, gate, state, dlast), ("dx", "dgate", "dstate")):
        oracle.within(got, value, off, name)
    for one, two in zip(grads, O.gated_scan_backward(dh, x, gate, starts, dlast)):
        assert torch.equal(one, two)


@pytest.mark.parametrize("shape", SCANS)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("state", [False, True])
def test_scan(shape, kind, state):
    b, t, d = shape
    x, gate, dh = normal(shape, kind, seed=30), gates(shape, kind, 31), normal(shape, kind, seed=32)
    check_scan(x, gate, normal((b, d), seed=33) if state else None, dh, normal((b, d), seed=34) if state else None)


@pytest.mark.parametrize("shape", [(1, 5000, 64), (1, 8209, 24), (3, 2049, 200), (2, 4111, 130)])
@pytest.mark.parametrize("kind", KINDS)
def test_long_sequences_are_spread_over_clusters(shape, kind):
    b, t, d = shape
    x, gate, dh = normal(shape, kind, seed=35), gates(shape, kind, 36), normal(shape, kind, seed=37)
    check_scan(x, gate, normal((b, d), seed=38), dh, normal((b, d), seed=39))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("layout", ["halves", "odd halves", "offset", "pad 2", "steps first", "expanded", "every second"])
@pytest.mark.parametrize("d", [64, 70, 33])
def test_scan_of_views(kind, layout, d):
    b, t = 3, 75
    if layout.endswith("halves"):
        both = normal((b, t, 2 * d + (layout == "odd halves")), kind, seed=40)
        x, gate = both[..., :d], both[..., d:2 * d]
    elif layout == "steps first":
        x, gate = normal((t, b, d), kind, seed=41).transpose(0, 1), normal((b, t, d), kind, seed=42)
    elif layout == "expanded":
        x, gate = normal((1, t, d), kind, seed=43).expand(b, t, d), normal((b, 1, d), kind, seed=44).expand(b, t, d)
    elif layout == "every second":
        x, gate = normal((b, t, 2 * d), kind, seed=45)[..., ::2], normal((b, 2 * t, d), kind, seed=46)[:, ::2]
    else:
        more = dict(offset=1) if layout == "offset" else dict(pad=2, offset=2)
        x, gate = normal((b, t, d), kind, seed=47, **more), normal((b, t, d), kind, seed=48, **more)
    dh = normal((t, b, d), kind, seed=49).transpose(0, 1)
    check_scan(x, gate, normal((b, d), seed=50), dh)


def test_gates_without_bound_keep_and_replace():
    shape = (2, 200, 70)
    x, gate, dh = normal(shape, seed=51), gates(shape, F32, 52), normal(shape, seed=53)
    gate[0, 50] = gate[1, 17] = -float("inf")                                      # a new sequence begins
    gate[:, 100:140] = float("inf")                                                # padding: the state stays
    state = normal((2, 70), seed=54)
    check_scan(x, gate, state, dh, normal((2, 70), seed=55))
    h, last, _ = O.gated_scan_forward(x, gate, state)
    # Step by step nothing changes; where a group of steps that are formed together ends, the state behind it is h + (B - C h), not what the last of its steps left: both are
    # the state within its error.  Where nothing but +infinity stands, B = C = 0, and the state stays to the last bit.
    assert ((h[:, 99:100] - h[:, 100:140]).abs() <= 2 * oracle.scan(x, gate, state)[1][:, 99:100] + h[:, 99:100].abs() * 2 * oracle.U32).all()
    for steps in (3, 200, 5000):
        held, last, _ = O.gated_scan_forward(normal((2, steps, 70), seed=56), torch.full((2, steps, 70), float("inf"), device="cuda"), state)
        assert torch.equal(last, state) and torch.equal(held, state[:, None].expand(2, steps, 70))
    flat = torch.full((1, 3000, 8), 40.0, device="cuda")
    held, _, _ = O.gated_scan_forward(normal((1, 3000, 8), seed=56), flat, state[:1, :8])
    assert (held - state[:1, None, :8]).abs().max() < 1e-12                         # z = 4e-18


def test_a_state_at_its_input_stays_there():
    """h = x is a fixed point to the last bit, however slowly the channel forgets."""
    x = normal((1, 1, 64), seed=57).expand(1, 40_000, 64).contiguous()
    gate = torch.linspace(-4.0, 12.0, 64, device="cuda").expand(1, 40_000, 64).contiguous()
    h, last, _ = O.gated_scan_forward(x, gate, x[:, 0].contiguous())
    assert (h - x).abs().max() <= 4 * oracle.U32 * float(x.abs().max())


@pytest.mark.parametrize("where", ["x", "gate"])
@pytest.mark.parametrize("kind", [F32, BF16])
def test_nan_stays_in_its_channel_and_behind_its_step(where, kind):
    shape = (2, 300, 66)
    x, gate, dh = normal(shape, kind, seed=58), gates(shape, kind, 59), normal(shape, kind, seed=60)
    clean = O.gated_scan_forward(x, gate)[0]
    (x if where == "x" else gate)[1, 150, 7] = float("nan")
    h, last, starts = O.gated_scan_forward(x, gate, None, keep=True)
    bad = torch.zeros(shape, dtype=torch.bool, device="cuda")
    bad[1, 150:, 7] = True
    assert torch.equal(torch.isnan(h), bad) and torch.equal(h[~bad], clean[~bad])
    dx, dgate, dstate = O.gated_scan_backward(dh, x, gate, starts)
    channel = torch.zeros(shape, dtype=torch.bool, device="cuda")
    channel[1, :, 7] = True
    assert torch.isfinite(dx[~channel]).all() and torch.isfinite(dgate[~channel]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", [(1, 1), (3, 64), (64, 1000), (5, 1001), (128, 24)])
def test_one_step(kind, shape):
    x, gate, state = normal(shape, kind, seed=61, pad=shape[-1]), gates(shape, kind, 62), normal(shape, seed=63)
    want, error, _, _, _ = oracle.scan(x[:, None], gate[:, None], state)
    out, kept_state = torch.empty_like(state), state.clone()
    h = O.gated_scan_step(x, gate, state, out=out)
    oracle.within(h, want[:, 0], error[:, 0])
    oracle.within(out, want[:, 0], error[:, 0])
    assert torch.equal(state, kept_state)
    version = state._version
    assert torch.equal(O.gated_scan_step(x, gate, state), h) and torch.equal(state, out) and state._version > version


def test_steps_one_by_one_are_the_scan():
    x, gate, state = normal((4, 40, 96), BF16, seed=64), gates((4, 40, 96), BF16, 65), normal((4, 96), seed=66)
    h, last, _ = O.gated_scan_forward(x, gate, state)
    want, error, _, last_error, _ = oracle.scan(x, gate, state)
    for t in range(40):
        oracle.within(O.gated_scan_step(x[:, t], gate[:, t], state), want[:, t], error[:, t])
    assert ((state - last).abs().double() <= 2 * last_error + last.abs() * 2 * oracle.U32).all()


def test_nothing_to_scan():
    state = normal((3, 10), seed=67)
    h, last, starts = O.gated_scan_forward(normal((3, 0, 10)), normal((3, 0, 10)), state, keep=True)
    assert h.shape == (3, 0, 10) and torch.equal(last, state)
    dlast = normal((3, 10), seed=68)
    dx, dgate, dstate = O.gated_scan_backward(h, h, h, starts, dlast)
    assert dx.shape == dgate.shape == (3, 0, 10) and torch.equal(dstate, dlast)
    h, last, starts = O.gated_scan_forward(normal((0, 5, 10)), normal((0, 5, 10)), None, keep=True)
    assert h.shape == (0, 5, 10) and last.shape == (0, 10)
    assert O.gated_scan_backward(h, h, h, starts)[2].shape == (0, 10)
    assert O.gated_scan_step(normal((0, 10)), normal((0, 10)), normal((0, 10))).shape == (0, 10)


def test_scan_gradients_are_those_of_differences():
    shape, step = (2, 37, 6), 2.0 ** -7
    x, gate, state = (normal(s, seed=70 + k).requires_grad_() for k, s in enumerate((shape, shape, (2, 6))))
    dh, dlast = normal(shape, seed=73), normal((2, 6), seed=74)
    h, last = O.gated_scan(x, gate, state)
    ((h * dh).sum() + (last * dlast).sum()).backward()
    for k, at in ((0, (1, 20, 3)), (1, (0, 5, 2)), (1, (1, 36, 0)), (2, (1, 4))):
        loss = []
        for sign in (1, -1):
            moved = [t.detach().double().clone() for t in (x, gate, state)]
            moved[k][at] += sign * step
            hs, _, l, _, _ = oracle.scan(*moved)
            loss.append(float((hs * dh).sum() + (l * dlast).sum()))
        # linear in x and state; in a gate the loss is c sigmoid: its third derivative is below |c| / 8, so the difference is off by at most step^2 / 48 |c|, |c| < 100
        assert abs((loss[0] - loss[1]) / (2 * step) - float((x, gate, state)[k].grad[at])) < 100 / 48 * step * step + 1e-4


def test_scan_is_differentiable_where_only_some_outputs_are_used():
    shape = (2, 50, 16)
    x, gate, state = normal(shape, seed=75).requires_grad_(), gates(shape, F32, 76).requires_grad_(), normal((2, 16), seed=77).requires_grad_()
    for use in ("h", "last"):
        h, last = O.gated_scan(x, gate, state)
        grads = torch.autograd.grad((h if use == "h" else last).sum(), (x, gate, state))
        want = oracle.scan_gradient(torch.full(shape, float(use == "h"), device="cuda"), x.detach(), gate.detach(), state.detach(), None if use == "h" else torch.ones(2, 16, device="cuda"))
        for got, (value, error) in zip(grads, want):
            oracle.within(got, value, error)
    with torch.no_grad():
        assert torch.equal(O.gated_scan(x, gate, state)[0], h)


# ------------------------------------------------------------------------------------------ streams, graphs

def all_of_them(rng, tokens, weight, gate, state):
    """A block as a network has it, and its gradients."""
    e = O.embedding(tokens, weight, 3.0)
    h, last = O.gated_scan(e, gate, state)
    d = O.dropout(h, 0.2, rng, 4, e)
    return (d, last, *torch.autograd.grad(d.float().sum() + last.sum(), (weight, gate, state)))


@pytest.mark.parametrize("steps", [60, 700])                                       # without and with a sort, a sequence whole and in segments
def test_a_run_of_them_captured_and_replayed_follows_its_inputs(steps):
    shape = (4, steps)
    tokens = tokens_for(4 * steps, 100, 80).view(shape)
    weight, gate, state = normal((100, 64), BF16, seed=81).requires_grad_(), gates((*shape, 64), BF16, 82).requires_grad_(), normal((4, 64), seed=83).requires_grad_()
    rng = rng_of(3, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_of_them(rng, tokens, weight, gate, state)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outputs = all_of_them(rng, tokens, weight, gate, state)
        rng[1] += 1
    for step in range(3):
        with torch.no_grad():
            weight.normal_(generator=gen(84 + step))
            tokens.copy_(tokens_for(4 * steps, 100, 90 + step).view(shape))
        want = all_of_them(rng_of(3, step), tokens, weight, gate, state)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(outputs, want)) and rng.tolist() == [3, step + 1]


@pytest.mark.parametrize("count", [500, 3000])
def test_a_captured_gradient_without_any_row_is_whole_before_what_follows(count):
    """No CTA of the summing kernels has work: what comes next in the graph still finds all zeros written."""
    tokens, dout = torch.full((count,), -100, device="cuda"), normal((count, 512), F32, seed=95)
    out = torch.empty(60_000, 512, device="cuda")
    O.embedding_backward(dout, tokens, 60_000, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O.embedding_backward(dout, tokens, 60_000, out=out)
        seen = out.clone()
    for _ in range(5):
        out.fill_(1.0)
        graph.replay()
        assert not seen.any()


@pytest.mark.parametrize("where", ["cpu", "type", "shape", "overlap"])
def test_refusals(where):
    x, state = normal((3, 8)), normal((3, 8))
    tokens, weight, rng = torch.zeros(3, dtype=torch.int64, device="cuda"), normal((5, 8)), rng_of(1, 2)
    scan = normal((2, 5, 8))
    calls = {
        "cpu": [lambda: O.embedding(tokens.cpu(), weight), lambda: O.embedding_backward(x, tokens.cpu(), 5), lambda: O.dropout(x, 0.1, rng.cpu()), lambda: O.gated_scan(scan, scan.cpu()),
                lambda: O.gated_scan(scan, scan, normal((2, 8)).cpu()), lambda: O.gated_scan_step(x, x, state.cpu())],
        "type": [lambda: O.embedding(tokens.float(), weight), lambda: O.embedding(tokens, weight.double()), lambda: O.embedding(tokens, weight, dtype=torch.int32), lambda: O.dropout(x, 0.1, rng.int()),
                 lambda: O.dropout(x, 0.1, rng, residual=x.half()), lambda: O.gated_scan(scan, scan.half()), lambda: O.gated_scan(scan, scan, normal((2, 8), F16)),
                 lambda: O.gated_scan_step(x, x.half(), state), lambda: O.embedding_backward(x, tokens, 5, out=torch.empty(5, 8, dtype=torch.int32, device="cuda"))],
        "shape": [lambda: O.embedding(tokens, weight[0]), lambda: O.embedding_backward(x, tokens[:2], 5), lambda: O.embedding_backward(x, tokens, 0), lambda: O.embedding_backward(x, tokens, 5, out=weight[:4]),
                  lambda: O.dropout(x, 0.1, rng, residual=x[:2]), lambda: O.dropout(x, 0.1, rng[:1]), lambda: O.gated_scan(scan, scan[:, :4]), lambda: O.gated_scan(x, x), lambda: O.gated_scan(scan, scan, state),
                  lambda: O.gated_scan_backward(scan, scan, scan, state), lambda: O.gated_scan_step(scan, scan, state), lambda: O.gated_scan_step(x, x, state.t())],
        "overlap": [lambda: O.embedding_backward(x, tokens[:3], 3, out=x), lambda: O.gated_scan_step(x, x, state, out=x), lambda: O.gated_scan_step(x, x.clone(), state.view(-1)[:24].view(3, 8), out=state.new_empty(0).view(0, 8))],
    }
    for call in calls[where]:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: O.dropout(x, 1.5, rng), lambda: O.dropout(x, float("nan"), rng), lambda: O.dropout(x, 0.1, rng, -1), lambda: O.dropout_backward(x.half(), 0.1, rng, dtype=F32)):
        with pytest.raises(B.ApmsError):
            call()


def test_calls_on_two_streams_do_not_meet():
    streams = [torch.cuda.Stream() for _ in range(2)]
    inputs = [(rng_of(k, 0), tokens_for(4 * 600, 3000, 85 + k).view(4, 600), normal((3000, 256), BF16, seed=86 + k).requires_grad_(), gates((4, 600, 256), BF16, 87 + k).requires_grad_(),
               normal((4, 256), seed=88 + k).requires_grad_()) for k in range(2)]
    want = [all_of_them(*i) for i in inputs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(all_of_them(*inputs[k]))
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(a, b) for run in got[k] for a, b in zip(run, want[k]))
