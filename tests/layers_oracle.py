"""Plain 64-bit forms of the layers' operators, with bounds on what 32-bit arithmetic may be off by."""
import numpy as np
import torch

U32 = 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}     # half the smallest subnormal


def within(got, want, error, what=""):
    """got is want, off by `error` and by its own type's rounding; NaN and infinities where want has them."""
    assert got.shape == want.shape, (got.shape, want.shape)
    g = got.double()
    top = torch.finfo(got.dtype).max
    odd = ~torch.isfinite(want) | (want.abs() > top)
    assert torch.equal(torch.isnan(g), torch.isnan(want)), f"{what}: NaN elsewhere"
    assert torch.equal(g[odd & ~torch.isnan(want)], want[odd & ~torch.isnan(want)].sign() * float("inf")), f"{what}: infinities"
    error = torch.as_tensor(error, device=want.device).expand(want.shape)
    bound = error + (want.abs() + error) * HALF_STEP[got.dtype] + LEAST[got.dtype]
    bad = ((g - want).abs() > bound) & ~odd
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, the worst {float(((g - want).abs() / bound)[bad].max()):.2f} of the bound"


# ------------------------------------------------------------------------------------------ embedding

def rows_of(tokens, vocabulary):
    return torch.where((tokens >= 0) & (tokens < vocabulary), tokens.long(), vocabulary)


def embedding(tokens, weight, scale):
    """Values, and what one product rounded to 32 bits (by a scale that was) may be off by."""
    table = torch.cat([weight.double(), weight.new_zeros(1, weight.shape[1], dtype=torch.float64)])
    v = table[rows_of(tokens, weight.shape[0])] * float(np.float32(scale))
    return v, v.abs() * U32


def embedding_gradient(dout, tokens, vocabulary, scale):
    """A sum of n values in any order is off by at most (n - 1) roundings of the sum of their sizes; one more for the scale."""
    at, d = rows_of(tokens, vocabulary).flatten(), dout.double().reshape(-1, dout.shape[-1])
    sums, sizes = (torch.zeros(vocabulary + 1, d.shape[1], dtype=torch.float64, device=d.device).index_add_(0, at, v) for v in (d, d.abs()))
    n = torch.bincount(at, minlength=vocabulary + 1).double()[:, None]
    scale = float(np.float32(scale))
    return (sums * scale)[:-1], (sizes * abs(scale) * (n - 1).clamp(min=0) * 1.001 * U32 + sums.abs() * abs(scale) * U32 * 1.001)[:-1]


# ------------------------------------------------------------------------------------------ dropout

def philox(counter, key, rounds):
    """Salmon et al., 2011, on numpy arrays of 64-bit integers."""
    word = np.uint64(0xFFFFFFFF)
    c, k = [np.asarray(v, dtype=np.uint64) for v in counter], [np.uint64(v) for v in key]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & word, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & word]
        k = [(k[0] + np.uint64(0x9E3779B9)) & word, (k[1] + np.uint64(0xBB67AE85)) & word]
    return c


def kept(n, p, seed, step, site):
    blocks = (n + 7) // 8
    words = philox([np.arange(blocks), np.full(blocks, site), np.full(blocks, step & 0xFFFFFFFF), np.full(blocks, (step >> 32) & 0xFFFFFFFF)],
                   [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF], 7)
    bits = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=1).ravel()[:n]
    border = int(np.floor(65536 * p + 0.5))
    return torch.from_numpy(bits >= border), 65536 / (65536 - border) if border < 65536 else 0.0


def dropout(x, p, seed, step, site, residual=None):
    """The scale, the product and the sum are each rounded once to 32 bits."""
    mask, scale = kept(x.numel(), p, seed, step, site)
    v = torch.where(mask.view(x.shape).to(x.device), x.double() * scale, 0.0)
    if residual is None:
        return v, v.abs() * 2.01 * U32
    h = v + residual.double()
    return h, v.abs() * 2.01 * U32 + h.abs() * U32


# ------------------------------------------------------------------------------------------ gated linear recurrence

def sigmoid_error(kind):
    """Relative error of z = 1 / (1 + exp(gate)) in units of 2^-24.  binary32: the power of two 4 (its documented 2^-22), the
    factor for its argument's rest 1, the sum 1, the reciprocal 2 (one unit in the last place).  16 bits, |gate| <= 16: the argument 1.5 |gate| = 24, the power of two 4, the
    sum 1, the reciprocal 2, and 3 to spare."""
    return 8.0 if kind == torch.float32 else 34.0


def scan(x, gate, state=None):
    """(h, error of h, last, error of last, and for the gradients z, a, h before each step).  With M the largest of |x| and |state| of a channel every difference and partial
    state is below 2 M; a step's own errors are below (2 z (sigmoid_error + 2) + 8) M units: z's, and those of the differences, of the step's sum and of the spans' joins."""
    b, t, d = x.shape
    x, g = x.double(), gate.double()
    a, z = torch.sigmoid(g), torch.sigmoid(-g)
    h = torch.zeros(b, d, dtype=torch.float64, device=x.device) if state is None else state.double()
    most = torch.cat([x.abs(), h.abs()[:, None]], 1).amax(1)
    error = torch.zeros_like(h)
    k = sigmoid_error(gate.dtype) + 2
    hs, errors, before, errors_before = [], [], [], []
    for i in range(t):
        before.append(h)
        errors_before.append(error)
        h = torch.where(z[:, i] == 1, x[:, i] + 0 * h, torch.where(z[:, i] == 0, h + 0 * x[:, i], a[:, i] * h + z[:, i] * x[:, i]))
        error = a[:, i] * error + (2 * z[:, i] * k + 8) * most * U32
        hs.append(h)
        errors.append(error)
    stack = lambda v: torch.stack(v, 1) if v else x.new_zeros(b, 0, d)
    return stack(hs), stack(errors), h, error, (z, a, stack(before), stack(errors_before))


def scan_gradient(dh, x, gate, state=None, dlast=None):
    """((dx, error), (dgate, error), (dstate, error)).  k = a G is off by a times G's error, by z's error times G and by the roundings of the sum and of the spans' joins;
    all partial sums are below the sum of the sizes."""
    b, t, d = x.shape
    _, _, _, _, (z, a, before, before_error) = scan(x, gate, state)
    units = sigmoid_error(gate.dtype) + 2
    k = torch.zeros(b, d, dtype=torch.float64, device=x.device) if dlast is None else dlast.double()
    size, error = k.abs(), torch.zeros_like(k)
    x, dh = x.double(), dh.double()
    dx, dx_error, dg, dg_error = ([None] * t for _ in range(4))
    for i in reversed(range(t)):
        g, size = dh[:, i] + k, dh[:, i].abs() + size
        error = error + 4 * size * U32
        zi, ai, e = z[:, i], a[:, i], before[:, i] - x[:, i]
        az = ai * zi
        dx[i], dx_error[i] = zi * g, zi * error + zi * size * (units + 1) * U32
        dg[i] = g * e * az
        dg_error[i] = az * (error * e.abs() + size * (before_error[:, i] + e.abs() * U32)) + dg[i].abs() * (2 * units + 4) * U32
        error = ai * error + size * (zi * units + 4) * U32
        k, size = ai * g, ai * size
    stack = lambda v: torch.stack(v, 1) if t else x.new_zeros(b, 0, d)
    return (stack(dx), stack(dx_error)), (stack(dg), stack(dg_error)), (k, error)
