"""What is measured of the operators that a residual network needs beside its norms: the embedding lookup with scaling and its
gradient, dropout at a residual junction (its mask a function of seed, step, site and index, never stored) and its gradient, and the gated
linear recurrence, its single-token form and its backward pass.

`run` is one pass: with `own` false in elementary torch operations in 32 bits, with `own` true through the package.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
MOST = 1 << 26                       # elements of the largest activation or table
SITE = 5                             # the dropout's place in its network
PHILOX_ROUNDS = 7


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # the next token's row, BERT-Large-shaped vocabulary and width: what a launch costs
        _embed("embed 1x1024 bf16", "embed", tokens=1, width=1024, vocab=30522, type="bf16", out="bf16", scale=32.0),
        # 32 sequences of 512 tokens, rows of a binary32 table scaled by sqrt(width) into bfloat16 activations
        _embed("embed 16384x1024 f32 to bf16", "embed", tokens=16384, width=1024, vocab=30522, type="f32", out="bf16", scale=32.0),
        # gradient of one sequence at BERT-Base's width, binary32: nearly all of the table's rows stay zero
        _embed("embed back 512x768 f32", "embed back", tokens=512, width=768, vocab=30522, type="f32", out="f32"),
        # gradient of 128 sequences of 512 tokens, an eighth of them padding, bfloat16 into the binary32 flat gradient
        _embed("embed back 65536x1024 bf16 to f32", "embed back", tokens=65536, width=1024, vocab=30522, type="bf16", out="f32", padding=0.125, scale=32.0),
        # one sequence at BERT-Base's width behind a sublayer
        _drop("drop 512x768 bf16", "drop", rows=512, width=768, type="bf16"),
        # a junction of the big batch: dropout and the addition to the residual stream
        _drop("drop add 16384x4096 bf16", "drop", rows=16384, width=4096, type="bf16", residual="same"),
        # the gradient that comes back from a binary32 stream, odd sizes, a padded buffer's rows
        _drop("drop back 7777x1001 f32 to bf16", "drop back", rows=7777, width=1001, type="bf16", residual="f32", pad=23),
        # 64 sequences' next token against their states
        _scan("step 64x4096 bf16", "step", batch=64, steps=1, width=4096, type="bf16"),
        # a few sequences of odd length and width in binary32, going on from a state
        _scan("scan 3x511x1001 f32", "scan", batch=3, steps=511, width=1001, type="f32", state=True),
        # one long sequence: little beside its length to spread the work over
        _scan("scan 1x32768x1024 bf16", "scan", batch=1, steps=32768, width=1024, type="bf16"),
        # a training batch, x and gate halves of one projection's output
        _scan("scan 8x4096x2048 bf16", "scan", batch=8, steps=4096, width=2048, type="bf16", joint=True),
        # and its backward pass
        _scan("scan back 8x4096x2048 bf16", "scan back", batch=8, steps=4096, width=2048, type="bf16", joint=True),
    ]


def _embed(name, op, tokens, width, vocab, type, out, scale=1.0, padding=0.0, skipped=0.0, index="i64"):
    """padding: the share of tokens that are 0; skipped: the share that is -100 (no row, no gradient)."""
    return {"name": name, "op": op, "tokens": tokens, "width": width, "vocab": vocab, "type": type, "out": out, "scale": scale,
            "padding": padding, "skipped": skipped, "index": index}


def _drop(name, op, rows, width, type, residual="none", p=0.1, pad=0):
    return {"name": name, "op": op, "rows": rows, "width": width, "type": type, "residual": residual, "p": p, "pad": pad}


def _scan(name, op, batch, steps, width, type, state=False, joint=False):
    """state: the recurrence goes on from one; joint: x and gate are halves of one tensor's rows."""
    return {"name": name, "op": op, "batch": batch, "steps": steps, "width": width, "type": type, "state": state, "joint": joint}


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    width = _log_uniform(rng, lo, hi)
    return max(lo, width // 64 * 64) if rng.random() < 0.6 else width


def draw(rng):
    family = rng.choice(["embed", "drop", "scan"])
    if family == "embed":
        width = _width(rng, 64, 8192)
        vocab = _log_uniform(rng, 100, min(262144, MOST // width))
        c = _embed("", rng.choice(["embed", "embed back"]), _log_uniform(rng, 1, min(131072, MOST // width)), width, vocab,
                   rng.choice(["f32", "bf16", "f16"]), rng.choice(["f32", "bf16", "f16"]), rng.choice([1.0, math.sqrt(width)]),
                   rng.choice([0.0, 0.0, 0.3]), rng.choice([0.0, 0.0, 0.15]), rng.choice(["i64", "i64", "i32"]))
    elif family == "drop":
        width = _width(rng, 64, 16384)
        c = _drop("", rng.choice(["drop", "drop", "drop back"]), _log_uniform(rng, 1, min(65536, MOST // width)), width, rng.choice(["f32", "bf16", "f16"]),
                  rng.choice(["none", "same", "f32"]), rng.choice([0.1, 0.1, 0.25, 0.5, 0.0]), rng.choice([0, 0, 0, 8, 3]))
    else:
        op = rng.choice(["scan", "scan", "scan back", "step"])
        width = _width(rng, 64, 8192)
        batch = _log_uniform(rng, 1, 512 if op == "step" else 32)
        steps = 1 if op == "step" else _log_uniform(rng, 1, max(1, min(32768 if op == "scan" else 8192, MOST // (width * batch))))
        c = _scan("", op, batch, steps, width, rng.choice(["f32", "bf16", "bf16", "f16"]), state=rng.random() < 0.5, joint=rng.random() < 0.5)
    del c["name"]
    return c


def _shares(case):
    """How often a token is each of the vocabulary's: falling with its number, as in text."""
    p = 1.0 / (np.arange(case["vocab"]) + 2.7)
    p *= (1.0 - case["padding"] - case["skipped"]) / p.sum()
    p[0] += case["padding"]
    return p


def work(case):
    if case["op"].startswith("embed"):
        n, used = case["tokens"], case["tokens"] * case["width"]
        index = 8 if case["index"] == "i64" else 4
        if case["op"] == "embed":
            distinct = float(-np.expm1(n * np.log1p(-np.minimum(_shares(case), 1.0 - 1e-12))).sum())
            return {"bytes": n * index + distinct * case["width"] * SIZE[case["type"]] + used * SIZE[case["out"]], "flops": used}
        return {"bytes": n * index + used * (1.0 - case["skipped"]) * SIZE[case["type"]] + case["vocab"] * case["width"] * SIZE[case["out"]], "flops": 2 * used}
    es = SIZE[case["type"]]
    if case["op"].startswith("drop"):
        n, rs = case["rows"] * case["width"], {"none": 0, "same": es, "f32": 4}[case["residual"]]
        return {"bytes": n * (es + (2 * rs or es)) if case["op"] == "drop" else n * ((rs or es) + es), "flops": 2 * n}
    state = 4 * case["batch"] * case["width"]
    n = case["batch"] * case["steps"] * case["width"]
    if case["op"] == "scan back":
        return {"bytes": 5 * n * es + (3 if case["state"] else 2) * state, "flops": 16 * n}
    return {"bytes": 3 * n * es + (2 if case["state"] or case["op"] == "step" else 1) * state, "flops": 8 * n}


# ------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"].startswith("embed"):
        return _prepare_embedding(case, gen)
    if case["op"].startswith("drop"):
        return _prepare_dropout(case, gen, seed)
    return _prepare_recurrence(case, gen)


def _normal(gen, shape, kind, scale=1.0, pad=0):
    """Gaussian values, the rows `pad` elements further apart than they are long."""
    t = torch.empty(*shape[:-1], shape[-1] + pad, dtype=kind, device="cuda")
    return t.normal_(0.0, scale, generator=gen)[..., :shape[-1]]


def _prepare_embedding(case, gen):
    n = case["tokens"]
    upto = torch.from_numpy(np.cumsum(_shares(case))).cuda()
    u = torch.empty(n, dtype=torch.float64, device="cuda").uniform_(generator=gen)
    tokens = torch.searchsorted(upto, u, right=True).clamp_(max=case["vocab"] - 1)
    tokens[u >= 1.0 - case["skipped"]] = -100
    state = {"case": case, "tokens": tokens if case["index"] == "i64" else tokens.int()}
    if case["op"] == "embed":
        state["weight"] = _normal(gen, (case["vocab"], case["width"]), TYPES[case["type"]], 0.02)
    else:
        state["dout"] = _normal(gen, (n, case["width"]), TYPES[case["type"]], 1e-2)
        state["out"] = torch.empty(case["vocab"], case["width"], dtype=TYPES[case["out"]], device="cuda")     # a place in the flat gradient
    return state


def _prepare_dropout(case, gen, seed):
    shape, kind = (case["rows"], case["width"]), TYPES[case["type"]]
    stream = torch.float32 if case["residual"] == "f32" else kind
    rng = random.Random(seed)
    state = {"case": case, "rng": torch.tensor([rng.getrandbits(62), rng.getrandbits(40)], device="cuda")}    # seed, step
    if case["op"] == "drop":
        state["x"] = _normal(gen, shape, kind, pad=case["pad"])
        state["residual"] = None if case["residual"] == "none" else _normal(gen, shape, stream, 2.0)
    else:
        state["dh"] = _normal(gen, shape, stream, 1e-2, pad=case["pad"])
    return state


def _prepare_recurrence(case, gen):
    """Gates whose channels forget over 2 to 1000 steps, with the spread that a projection gives them."""
    b, t, d, kind = case["batch"], case["steps"], case["width"], TYPES[case["type"]]
    shape = (b, d) if case["op"] == "step" else (b, t, d)
    bias = torch.empty(d, device="cuda").uniform_(0.0, 6.9, generator=gen).to(kind)
    if case["joint"]:
        x, gate = _normal(gen, (*shape[:-1], 2 * d), kind).chunk(2, -1)
    else:
        x, gate = _normal(gen, shape, kind), _normal(gen, shape, kind)
    gate += bias
    state = {"case": case, "x": x, "gate": gate, "state": None}
    if case["state"] or case["op"] == "step":
        state["state"] = _normal(gen, (b, d), torch.float32)
    if case["op"] == "step":
        state["next"] = torch.empty(b, d, device="cuda")
    if case["op"] == "scan back":
        state["dh"] = _normal(gen, shape, kind, 1e-2)
        state["dlast"] = _normal(gen, (b, d), torch.float32, 1e-2)
        if own:
            from paper_2008_11343_b200 import operators
            state["starts"] = operators.gated_scan_forward(x, gate, state["state"], keep=True)[2]      # what the forward pass leaves
    return state


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    case = state["case"]
    if own:
        return _run_own(case, state)
    return {"embed": _embedding, "embed back": _embedding_backward, "drop": _dropout, "drop back": _dropout_backward, "step": _step,
            "scan": _recurrence, "scan back": _recurrence_backward}[case["op"]](case, state)


def _run_own(case, s):
    from paper_2008_11343_b200 import operators
    op = case["op"]
    if op == "embed":
        return operators.embedding_forward(s["tokens"], s["weight"], case["scale"], dtype=TYPES[case["out"]])
    if op == "embed back":
        return operators.embedding_backward(s["dout"], s["tokens"], case["vocab"], case["scale"], out=s["out"])
    if op == "drop":
        return operators.dropout_forward(s["x"], case["p"], s["rng"], SITE, s["residual"])[0]
    if op == "drop back":
        return operators.dropout_backward(s["dh"], case["p"], s["rng"], SITE, dtype=TYPES[case["type"]])
    if op == "step":
        return operators.gated_scan_step(s["x"], s["gate"], s["state"], out=s["next"]), s["next"]
    if op == "scan":
        return operators.gated_scan_forward(s["x"], s["gate"], s["state"])[:2]
    dx, dgate, dstate = operators.gated_scan_backward(s["dh"], s["x"], s["gate"], s["starts"], s["dlast"])
    return (dx, dgate, dstate) if case["state"] else (dx, dgate)


def _embedding(case, s):
    known = (s["tokens"] >= 0) & (s["tokens"] < case["vocab"])
    rows = s["weight"][torch.where(known, s["tokens"], 0)].float() * case["scale"]
    return torch.where(known[:, None], rows, 0.0).to(TYPES[case["out"]])


def _embedding_backward(case, s):
    known = (s["tokens"] >= 0) & (s["tokens"] < case["vocab"])
    dweight = torch.zeros(case["vocab"], case["width"], device="cuda")
    dweight.index_add_(0, torch.where(known, s["tokens"], 0), torch.where(known[:, None], s["dout"].float(), 0.0))
    s["out"].copy_(dweight * case["scale"])
    return s["out"]


def _kept(case, rng):
    """Where the mask keeps, and what the kept are multiplied by.  Eight elements take one block of Philox 4x32 (Salmon et al., 2011):
    key = seed, counter = (number of the eight, site, step's low and high word); each of its four words gives two elements 16 bits, the low
    half first; an element is kept where they reach p * 2^16."""
    n, low = case["rows"] * case["width"], 0xFFFFFFFF
    c = [torch.arange((n + 7) // 8, device="cuda"), torch.full((1,), SITE, device="cuda"), rng[1] & low, (rng[1] >> 32) & low]
    key = [rng[0] & low, (rng[0] >> 32) & low]
    for _ in range(PHILOX_ROUNDS):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & low) ^ c[1] ^ key[0], b & low, ((a >> 32) & low) ^ c[3] ^ key[1], a & low]
        key = [(key[0] + 0x9E3779B9) & low, (key[1] + 0xBB67AE85) & low]
    bits = torch.stack([half for word in c for half in (word.expand(c[0].shape) & 0xFFFF, word.expand(c[0].shape) >> 16)], dim=1)
    border = math.floor(case["p"] * 65536 + 0.5)
    return (bits.flatten()[:n] >= border).view(case["rows"], case["width"]), 65536.0 / (65536 - border)


def _dropout(case, s):
    kept, scale = _kept(case, s["rng"])
    h = torch.where(kept, s["x"].float() * scale, 0.0)
    if s["residual"] is None:
        return h.to(s["x"].dtype)
    return (h + s["residual"].float()).to(s["residual"].dtype)


def _dropout_backward(case, s):
    kept, scale = _kept(case, s["rng"])
    return torch.where(kept, s["dh"].float() * scale, 0.0).to(TYPES[case["type"]])


def _step(case, s):
    taken = torch.sigmoid(-s["gate"].float())
    torch.add(s["state"], taken * (s["x"].float() - s["state"]), out=s["next"])
    return s["next"].to(s["x"].dtype), s["next"]


def _states(case, s):
    """z = sigmoid(-gate) and the states h_t = h_(t-1) + z_t (x_t - h_(t-1)), the first of them before the first step; steps first."""
    x, z = s["x"].float().transpose(0, 1), torch.sigmoid(-s["gate"].float()).transpose(0, 1)
    h = torch.zeros(case["steps"] + 1, case["batch"], case["width"], device="cuda")
    if s["state"] is not None:
        h[0] = s["state"]
    for t in range(case["steps"]):
        torch.addcmul(h[t], z[t], x[t] - h[t], out=h[t + 1])
    return z, h


def _recurrence(case, s):
    _, h = _states(case, s)
    return h[1:].transpose(0, 1).to(s["x"].dtype), h[-1]


def _recurrence_backward(case, s):
    z, h = _states(case, s)
    a = torch.sigmoid(s["gate"].float()).transpose(0, 1)
    x, dh = s["x"].float().transpose(0, 1), s["dh"].float().transpose(0, 1)
    g = torch.empty_like(x)
    later = s["dlast"]
    for t in reversed(range(case["steps"])):
        torch.add(dh[t], later, out=g[t])
        later = a[t] * g[t]
    dx, dgate = (z * g).to(s["x"].dtype), (g * (h[:-1] - x) * a * z).to(s["x"].dtype)
    out = dx.transpose(0, 1), dgate.transpose(0, 1)
    return (*out, later) if case["state"] else out


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("embed"):
        return _exact_embedding(case, s)
    if case["op"].startswith("drop"):
        return _exact_dropout(case, s)
    return _exact_recurrence(case, s)


def _exact_embedding(case, s):
    outside = torch.logical_or(s["tokens"] < 0, s["tokens"] >= case["vocab"])
    tokens = s["tokens"].long().masked_fill(outside, case["vocab"])
    if case["op"] == "embed":
        table = torch.cat([s["weight"].double(), torch.zeros(1, case["width"], dtype=torch.float64, device="cuda")])
        return table.index_select(0, tokens).mul_(case["scale"])
    sums = torch.zeros(case["vocab"] + 1, case["width"], dtype=torch.float64, device="cuda")
    for part in range(0, case["tokens"], 8192):
        sums.index_put_((tokens[part:part + 8192],), s["dout"][part:part + 8192].double(), accumulate=True)
    return sums[:-1] * case["scale"]


def _product(a, m):
    """The high and low 32 bits of a * m, by 16-bit halves of m."""
    low, high = a * (m & 0xFFFF), a * (m >> 16)                     # below 2^48 each
    middle = (low >> 16) + (high & 0xFFFF)
    return (high >> 16) + (middle >> 16), ((middle & 0xFFFF) << 16) | (low & 0xFFFF)


def _exact_dropout(case, s):
    seed, step = (int(v) for v in s["rng"])
    n, word = case["rows"] * case["width"], 2 ** 32
    w = torch.zeros(-(-n // 8), 4, dtype=torch.int64, device="cuda")
    w[:, 0] = torch.arange(w.shape[0], device="cuda")
    w[:, 1], w[:, 2], w[:, 3] = SITE, step % word, step // word
    for r in range(PHILOX_ROUNDS):
        high0, low0 = _product(w[:, 0], 3528531795)
        high1, low1 = _product(w[:, 2], 3449720151)
        k0, k1 = (seed + r * 2654435769) % word, (seed // word + r * 3144134277) % word
        w = torch.stack([high1 ^ w[:, 1] ^ k0, low1, high0 ^ w[:, 3] ^ k1, low0], dim=1)
    bits = torch.stack([w % 65536, w // 65536], dim=2).view(-1)[:n]
    border = round(case["p"] * 65536 + 1e-9)
    x = (s["x"] if case["op"] == "drop" else s["dh"]).double().reshape(-1)
    h = (x * (bits >= border) * (65536 / (65536 - border))).view(case["rows"], case["width"])
    return h if case["op"] == "drop back" or s["residual"] is None else h + s["residual"].double()


def _doubled(a, b):
    """v_t = a_t v_(t-1) + b_t from v = 0 along the first dimension, by spans of doubling length."""
    span = 1
    while span < a.shape[0]:
        b = torch.cat([b[:span], b[span:] + a[span:] * b[:-span]])
        a = torch.cat([a[:span], a[span:] * a[:-span]])
        span *= 2
    return b


def _exact_recurrence(case, s):
    b, d = case["batch"], case["width"]
    parts = []
    for columns in torch.arange(d).split(max(1, (1 << 24) // (b * case["steps"]))):       # channels are independent
        c = slice(int(columns[0]), int(columns[-1]) + 1)
        x, gate = (s[k].double().reshape(b, case["steps"], d)[:, :, c].transpose(0, 1) for k in ("x", "gate"))
        a, z = 1 / (1 + torch.exp(-gate)), 1 / (1 + torch.exp(gate))
        first = torch.zeros(b, x.shape[2], dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()[:, c]
        taken = z * x
        taken[0] += a[0] * first
        h = _doubled(a, taken)
        if case["op"] != "scan back":
            parts.append((h.transpose(0, 1), h[-1]))
            continue
        g = s["dh"].double()[:, :, c].transpose(0, 1).clone()
        g[-1] += s["dlast"].double()[:, c]
        g = _doubled(torch.cat([torch.ones_like(a[:1]), a[1:].flip(0)]), g.flip(0)).flip(0)
        before = torch.cat([first[None], h[:-1]])
        parts.append(((z * g).transpose(0, 1), (g * (before - x) * a * z).transpose(0, 1), a[0] * g[0]))
    out = [torch.cat(p, dim=-1) for p in zip(*parts)]
    if case["op"] == "step":
        return out[0][:, 0], out[1]
    return tuple(out) if case["op"] == "scan" or case["state"] else tuple(out[:2])
