"""What is measured of the operators beside the compressed step: the gradient norm over a model's tensors, clipping
them into the flat vector a step takes, the root-mean-square norm at a residual junction (16/32-bit output, and 8-bit
output with scales) and its backward pass.

`run` is one pass: with `own` false in elementary torch operations in 32 bits, with `own` true through the package.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
E4M3_MAX = 448.0
MOST_GRADIENT = 335_141_888          # elements of the largest list: the BERT-Large-shaped parameter set
MOST_ACTIVATION = 16384 * 4096       # elements of the largest activation


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # a worker's gradients, BERT-Large-shaped set in binary32 (the benchmark's headline set), separate tensors
        _grads("norm bert-large f32", "norm", tensors="bert", layers=24, hidden=1024, ffn=4096, type="f32"),
        # the 64 tensors of log-uniform size of the benchmark's second set; matrices in bfloat16, every third tensor in binary32
        _grads("norm 64 mixed", "norm", tensors="random", count=64, total=1 << 24, type="mixed"),
        # a small fine-tuned head: few small tensors, the launch counts
        _grads("clip 6 small bf16", "clip", tensors="random", count=6, total=40_007, type="bf16", out="bf16"),
        # tensors that are views at odd offsets of one bucket, odd sizes, widened into a binary32 flat gradient
        _grads("clip 301 odd f16 bucket", "clip", tensors="random", count=301, total=20_000_003, type="f16", out="f32", bucket=True),
        # a worker's gradients, twelve encoder layers of width 1024 and the embeddings, bfloat16 in and out (16-bit training)
        _grads("clip bert 12x1024 bf16", "clip", tensors="bert", layers=12, hidden=1024, ffn=4096, type="bf16", out="bf16"),
        # the headline set, binary32 in and out
        _grads("clip bert-large f32", "clip", tensors="bert", layers=24, hidden=1024, ffn=4096, type="f32", out="f32"),
        # one token through a junction of width 1024: what a launch costs
        _rms("rms 1x1024 bf16", "rms", rows=1, width=1024, type="bf16", residual="same"),
        # a batch of 16 sequences of 512 tokens at the FFN's width
        _rms("rms 8192x4096 bf16", "rms", rows=8192, width=4096, type="bf16", residual="same"),
        # 8-bit output for the next matrix product: a scale per 128 columns, ragged rows and width, binary32 residual stream
        _rms("rms8 777x1000 bf16", "rms", rows=777, width=1000, type="bf16", residual="f32", weight="f32", group=128),
        # 8-bit output, a scale per token
        _rms("rms8 16384x4096 bf16", "rms", rows=16384, width=4096, type="bf16", residual="same", group=0),
        # backward of one sequence at BERT-Base's width, binary32
        _rms("back 512x768 f32", "back", rows=512, width=768, type="f32", residual="same"),
        # backward of the big batch, bfloat16, with the gradient that arrives on the residual stream
        _rms("back 16384x4096 bf16", "back", rows=16384, width=4096, type="bf16", residual="same"),
    ]


def _grads(name, op, tensors, type, count=0, total=0, layers=0, hidden=0, ffn=0, out="", bucket=False, layout=7, max_norm=1.0):
    return {"name": name, "op": op, "tensors": tensors, "count": count, "total": total, "layers": layers, "hidden": hidden,
            "ffn": ffn, "type": type, "out": out, "bucket": bucket, "layout": layout, "max_norm": max_norm}


def _rms(name, op, rows, width, type, residual, weight="same", group=-1, pad=0):
    return {"name": name, "op": op, "rows": rows, "width": width, "type": type, "residual": residual, "weight": weight,
            "group": group, "pad": pad}


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    if rng.random() < 0.5:
        total = _log_uniform(rng, 20_000, MOST_GRADIENT)
        c = _grads("", rng.choice(["norm", "clip"]), "random", rng.choice(["f32", "bf16", "f16", "mixed"]),
                   count=min(_log_uniform(rng, 1, 600), total), total=total, bucket=rng.random() < 0.3,
                   layout=rng.randrange(1 << 30), max_norm=rng.choice([1.0, 1.0, 1e4]))
        if c["op"] == "clip":
            c["out"] = rng.choice(["f32", "bf16", "f16"])
    else:
        width = _log_uniform(rng, 64, 16384)
        if rng.random() < 0.6:
            width = max(64, width // 64 * 64)          # what models use; the rest stays odd
        rows = _log_uniform(rng, 1, min(65536, MOST_ACTIVATION // width))
        kind = rng.choice(["f32", "bf16", "bf16", "f16"])
        c = _rms("", rng.choice(["rms", "rms", "back"]), rows, width, kind, rng.choice(["none", "same", "same", "f32"]),
                 weight=rng.choice(["same", "f32"]), pad=rng.choice([0, 0, 0, 8, 24, 3]))
        if c["op"] == "rms":
            c["group"] = rng.choice([-1, 0, 128])
    del c["name"]
    return c


def _sizes(case):
    """Element counts of the list's tensors."""
    if case["tensors"] == "bert":
        h, f = case["hidden"], case["ffn"]
        layer = [h * h, h] * 4 + [h, h, h * f, f, f * h, h, h, h]
        return [30522 * h, 512 * h, 2 * h, h, h] + layer * case["layers"] + [h * h, h]
    rng = random.Random(case["layout"])
    raw = [math.exp(rng.uniform(0.0, math.log(256.0))) for _ in range(case["count"])]
    unit = case["total"] / sum(raw)
    sizes = [max(1, int(r * unit)) for r in raw]
    sizes[-1] = max(1, sizes[-1] + case["total"] - sum(sizes))
    return sizes


def _types(case, count):
    return [("f32" if k % 3 == 2 else "bf16") if case["type"] == "mixed" else case["type"] for k in range(count)]


def work(case):
    if case["op"] in ("norm", "clip"):
        sizes = _sizes(case)
        read = sum(n * SIZE[t] for n, t in zip(sizes, _types(case, len(sizes))))
        n = sum(sizes)
        if case["op"] == "norm":
            return {"bytes": read + 4 * (len(sizes) + 1), "flops": 2 * n}
        return {"bytes": read + n * SIZE[case["out"]] + 4, "flops": 3 * n}
    n, es = case["rows"] * case["width"], SIZE[case["type"]]
    rs = {"none": 0, "same": es, "f32": 4}[case["residual"]]
    ws = 4 if case["weight"] == "f32" else es
    if case["op"] == "rms":
        out = es if case["group"] < 0 else 1
        groups = 0 if case["group"] < 0 else 1 if case["group"] == 0 else -(-case["width"] // case["group"])
        return {"bytes": n * (es + 2 * rs + out) + ws * case["width"] + 4 * case["rows"] * (1 + groups), "flops": 6 * n}
    hs = rs or es
    return {"bytes": n * (es + hs + es + rs + (rs if rs != es else 0)) + 2 * ws * case["width"] + 4 * case["rows"], "flops": 12 * n}


# ------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] in ("norm", "clip"):
        return _prepare_gradients(case, seed, gen)
    return _prepare_activations(case, gen)


def _prepare_gradients(case, seed, gen):
    """Gaussian gradients whose scale varies over three decades from tensor to tensor, as real layers' do."""
    sizes = _sizes(case)
    types = [TYPES[t] for t in _types(case, len(sizes))]
    rng = random.Random(seed)
    if case["bucket"]:                        # views of one buffer per type, one after the other: odd element offsets
        buckets = {t: torch.empty(1 + sum(n for n, u in zip(sizes, types) if u == t), dtype=t, device="cuda") for t in set(types)}
        at, tensors = {t: 1 for t in buckets}, []
        for n, t in zip(sizes, types):
            tensors.append(buckets[t][at[t]:at[t] + n])
            at[t] += n
    else:
        tensors = [torch.empty(n, dtype=t, device="cuda") for n, t in zip(sizes, types)]
    for t in tensors:
        t.normal_(0.0, math.exp(rng.uniform(math.log(1e-4 if t.dtype == torch.float16 else 1e-5), math.log(1e-2))), generator=gen)
    state = {"case": case, "tensors": tensors}
    if case["op"] == "clip":
        state["flat"] = torch.empty(sum(sizes), dtype=TYPES[case["out"]], device="cuda")
    if own:
        from paper_2008_11343_b200 import operators
        state["list"] = operators.TensorList(tensors)
    return state


def _prepare_activations(case, gen):
    """Activations with a few columns larger than the others, as trained models have; rows `pad` elements apart."""
    rows, width, kind = case["rows"], case["width"], TYPES[case["type"]]
    rkind = torch.float32 if case["residual"] == "f32" else kind
    wkind = torch.float32 if case["weight"] == "f32" else kind

    def normal(dtype, scale=1.0, pad=0):
        t = torch.empty(rows, width + pad, dtype=dtype, device="cuda")
        return t.normal_(0.0, scale, generator=gen)[:, :width]

    columns = torch.exp(0.5 * torch.empty(width, device="cuda").normal_(generator=gen))
    weight = (1.0 + 0.1 * torch.empty(width, device="cuda").normal_(generator=gen)).to(wkind)
    state = {"case": case, "weight": weight}
    if case["op"] == "rms":
        state["x"] = normal(kind, pad=case["pad"])
        state["x"] *= columns.to(kind)
        state["residual"] = None if case["residual"] == "none" else normal(rkind, 2.0)
        return state
    state["h"] = normal(kind if case["residual"] == "none" else rkind, 2.0)
    state["h"] *= columns.to(state["h"].dtype)
    state["rstd"] = torch.rsqrt((state["h"].double().square().sum(1) / width + EPS)).float()
    state["dy"] = normal(kind, 1e-2, pad=case["pad"])
    state["dh"] = None if case["residual"] == "none" else normal(rkind, 1e-2)
    return state


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    case = state["case"]
    if own:
        return _run_own(case, state)
    return {"norm": _norm, "clip": _clip, "rms": _rms_norm, "back": _rms_norm_backward}[case["op"]](case, state)


def _run_own(case, s):
    from paper_2008_11343_b200 import operators
    if case["op"] == "norm":
        return s["list"].grad_norm(s["tensors"])
    if case["op"] == "clip":
        return s["flat"], s["list"].clip_grads(s["tensors"], case["max_norm"], out=s["flat"])
    if case["op"] == "back":
        return operators.rms_norm_backward(s["dy"], s["h"], s["weight"], s["rstd"], dh=s["dh"])
    if case["group"] < 0:
        return operators.rms_norm_forward(s["x"], s["weight"], s["residual"], eps=EPS)
    return operators.rms_norm_fp8(s["x"], s["weight"], s["residual"], eps=EPS, group=case["group"])


def _norm(case, s):
    squares = torch.stack([t.float().square().sum() for t in s["tensors"]])
    return squares.sum().sqrt(), squares.sqrt()


def _clip(case, s):
    flat = torch.cat([t.float() for t in s["tensors"]])
    norm = flat.square().sum().sqrt()
    factor = torch.where(norm <= case["max_norm"], torch.ones_like(norm), case["max_norm"] / norm)
    s["flat"].copy_(flat * factor)
    return s["flat"], norm


def _rms_norm(case, s):
    x, r, w = s["x"], s["residual"], s["weight"].float()
    h = x.float() if r is None else x.float() + r.float()
    rstd = torch.rsqrt(h.square().sum(1) / case["width"] + EPS)
    y = h * rstd[:, None] * w
    kept = x if r is None else h.to(r.dtype)
    if case["group"] < 0:
        return y.to(x.dtype), kept, rstd
    q, scale = _to_e4m3(y, case)
    return q.to(torch.float8_e4m3fn), scale, kept, rstd


def _to_e4m3(y, case):
    """y over its group's scale, and the scales: a group is a row, or `group` columns of it."""
    rows, width = y.shape
    size = case["group"] or width
    groups = -(-width // size)
    padded = torch.zeros(rows, groups * size, dtype=y.dtype, device=y.device)
    padded[:, :width] = y
    padded = padded.view(rows, groups, size)
    most = padded.abs().amax(2)
    inverse = torch.where(most > 0, E4M3_MAX / most, torch.zeros_like(most))
    return (padded * inverse[:, :, None]).view(rows, groups * size)[:, :width], most / E4M3_MAX


def _rms_norm_backward(case, s):
    dy, h, w, rstd = s["dy"].float(), s["h"].float(), s["weight"].float(), s["rstd"][:, None]
    xhat = h * rstd
    a = dy * w
    dx = rstd * (a - xhat * ((a * xhat).sum(1, keepdim=True) / case["width"]))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    dw = (dy * xhat).sum(0).to(s["weight"].dtype)
    if s["dh"] is not None and s["dh"].dtype != s["dy"].dtype:
        return dx.to(s["dy"].dtype), dw, dx.to(s["dh"].dtype)
    return dx.to(s["dy"].dtype), dw


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        norms = torch.stack([torch.linalg.vector_norm(t, dtype=torch.float64) for t in s["tensors"]])
        return torch.linalg.vector_norm(norms), norms
    if case["op"] == "clip":
        flat = torch.cat([t.double() for t in s["tensors"]])
        norm = torch.linalg.vector_norm(flat)
        return flat * min(1.0, case["max_norm"] / float(norm)), norm
    w, width = s["weight"].double(), case["width"]
    if case["op"] == "rms":
        h = s["x"].double() + (0.0 if s["residual"] is None else s["residual"].double())
        rstd = (h.pow(2).mean(dim=1) + EPS).pow(-0.5)
        y = torch.einsum("rc,r,c->rc", h, rstd, w)
        if case["group"] < 0:
            return y, h, rstd
        size = case["group"] or width
        parts = [p for p in y.split(size, dim=1)]
        scales = torch.stack([p.abs().max(dim=1).values / E4M3_MAX for p in parts], dim=1)
        return torch.cat([p / k[:, None] for p, k in zip(parts, scales.unbind(1))], dim=1), scales, h, rstd
    dy, h, r = s["dy"].double(), s["h"].double(), s["rstd"].double()
    a = dy * w
    inner = torch.einsum("rc,rc->r", a, h) * r.pow(3) / width
    dx = a * r[:, None] - h * inner[:, None]
    if s["dh"] is not None:
        dx = dx + s["dh"].double()
    dw = torch.einsum("rc,rc,r->c", dy, h, r)
    if s["dh"] is not None and s["dh"].dtype != s["dy"].dtype:
        return dx, dw, dx
    return dx, dw
