"""Launch ONE kernel of the library a few times on a small case, for a profiler to capture.

    python -m paper_2008_11343_b200.profile_kernels --kernel k_apply [--d 33554432] [--n 8] [--launches 3]

Every kernel of the library can be reached by name; the case (d = 2^25 elements of the BERT-Large-shaped
set, n = 8 workers unless the kernel needs otherwise) is larger than L2 and holds a few GB on the device,
so that a capture of a handful of counters ends by itself in seconds.  The module only calls the public
binding; it computes nothing itself.  Prints one line per kernel with the CUDA-event time per launch and
the bytes the launch has to move, so that the same command is useful without a profiler too.
"""
from __future__ import annotations

import argparse
import itertools
import json
import sys


def _setup(d, n, chunk, compressor=None, variant=None, team=None, first_step=False, grad_dtype="float32", steps=1):
    import torch

    from . import binding as B
    from . import workloads as wl

    w = wl.sliced(wl.config(3), d).with_(n=n, chunk=chunk)
    ctx = B.Context(w.d, w.n, w.beta1, w.beta2, w.eps, w.lr, w.chunk)
    if compressor is not None:
        ctx.set_compressor(B.COMPRESSOR_TOPK, compressor)
    if variant is not None:
        ctx.set_variant(variant)
    if team is not None:
        ctx.set_team_mode(team)
    x0 = torch.empty(w.d, dtype=torch.float32, device="cuda").normal_(0.0, w.x0_std)
    ctx.set_params(x0)
    dt = getattr(torch, grad_dtype)
    grads = []
    for i in range(n):
        g = torch.empty(w.d, dtype=torch.float32, device="cuda")
        wl.device_gradient(w, 0, i, g)
        grads.append(g if dt == torch.float32 else g.to(dt))
    ctx.warmup_step(grads)
    ctx.warmup_step(grads)
    ctx.freeze_v()
    if not first_step:
        for _ in range(steps):              # the first step of the phase reads the binary32 momentum: not the steady state
            ctx.compressed_step(grads)      # (top-k: the predicted-threshold routes need a few steps of history)
    torch.cuda.synchronize()
    return ctx, w, grads


# kernel name -> (what to set up, what to call per launch, which timer of the library sees it)
def _cases(args):
    from . import binding as B

    d, n = args.d, args.n
    return {
        "k_warmup_adam": dict(setup=dict(chunk=32768), phase="warmup", timer=B.KERNEL_WARMUP_ADAM,
                              bytes=lambda w: (4 * w.n + 24) * w.d),
        "k_worker_fine": dict(setup=dict(chunk=32768), call="worker_phase", timer=B.KERNEL_WORKER,
                              bytes=lambda w: w.n * (12 * w.d + w.d // 8) + w.d // 8),
        "k_worker_fine_split": dict(setup=dict(chunk=32768 + 32), call="worker_phase", timer=B.KERNEL_WORKER,
                                    bytes=lambda w: w.n * (12 * w.d + w.d // 8) + w.d // 8),
        "k_worker_fine_bf16": dict(setup=dict(chunk=32768, grad_dtype="bfloat16"), call="worker_phase", timer=B.KERNEL_WORKER,
                                   bytes=lambda w: w.n * (10 * w.d + w.d // 8) + w.d // 8),
        "k_worker_fine_words": dict(setup=dict(chunk=128), call="worker_phase", timer=B.KERNEL_WORKER,
                                    bytes=lambda w: w.n * (12 * w.d + w.d // 8) + w.d // 8),
        "k_finalize_words": dict(setup=dict(chunk=128), call="worker_phase", timer=B.KERNEL_WORKER,
                                 bytes=lambda w: w.n * (8 * (w.d // 32) + 4 * w.n_chunks)),
        "k_worker": dict(setup=dict(chunk=160, team=B.TEAM_WARP), call="worker_phase", timer=B.KERNEL_WORKER,
                         bytes=lambda w: w.n * (12 * w.d + w.d // 8) + w.d // 8),
        "k_worker_m32": dict(setup=dict(chunk=32768, first_step=True), call="first_worker_phase", timer=B.KERNEL_WORKER,
                             bytes=lambda w: w.n * (12 * w.d + w.d // 8) + 4 * w.d),
        "k_finalize_fine": dict(setup=dict(chunk=32768), call="worker_phase", timer=B.KERNEL_WORKER,
                                bytes=lambda w: w.n * (8 * (w.d // 512) + 4 * w.n_chunks)),
        "k_server_staged": dict(setup=dict(chunk=32768), call="step", timer=B.KERNEL_SERVER,
                                bytes=lambda w: w.n * w.d // 8 + 8 * w.d + w.d // 8 + 12 * w.d),
        "k_server_staged_unfused": dict(setup=dict(chunk=4 * 65536), call="worker_phase", timer=B.KERNEL_SERVER,
                                        bytes=lambda w: w.n * w.d // 8 + 8 * w.d + w.d // 8),
        "k_server_staged_lagged": dict(setup=dict(chunk=4 * 65536), call="step", timer=B.KERNEL_SERVER,
                                       bytes=lambda w: w.n * w.d // 8 + 8 * w.d + w.d // 4 + 12 * w.d),
        "k_server_packed": dict(setup=dict(chunk=1024), call="step", timer=B.KERNEL_SERVER,
                                bytes=lambda w: w.n * w.d // 8 + 8 * w.d + w.d // 8 + 12 * w.d),
        "k_server": dict(setup=dict(chunk=160), call="step", timer=B.KERNEL_SERVER,
                         bytes=lambda w: w.n * w.d // 8 + 8 * w.d + w.d // 8),
        "k_apply": dict(setup=dict(chunk=160), call="step", timer=B.KERNEL_APPLY,
                        bytes=lambda w: 12 * w.d + w.d // 8),
        "k_make_den": dict(setup=dict(chunk=32768, first_step=True), call="make_den", timer=None,
                           bytes=lambda w: 8 * w.d),
        "k_apply_gradient": dict(setup=dict(chunk=32768, variant=B.VARIANT_GRADIENT), call="step", timer=B.KERNEL_APPLY,
                                 bytes=lambda w: 20 * w.d + w.d // 8),
        "k_uncompressed": dict(setup=dict(chunk=32768), call="uncompressed", timer=B.KERNEL_WARMUP_ADAM,
                               bytes=lambda w: (4 * w.n + 20) * w.d),
        "k_noalloc_compress": dict(setup=None, call="noalloc", timer=None, bytes=lambda w: 4 * w.d + w.d // 8),
        "k_topk_worker": dict(setup=dict(chunk=32768, compressor=0.01), call="step", timer=B.KERNEL_WORKER,
                              bytes=lambda w: w.n * (12 * w.d + w.d // 4) + 4 * w.d),
        "k_topk_server": dict(setup=dict(chunk=32768, compressor=0.01), call="step", timer=B.KERNEL_SERVER,
                              bytes=lambda w: w.n * (w.d // 8 + int(0.04 * w.d)) + 24 * w.d + w.d // 8),
        "k_topk_worker_band": dict(setup=dict(chunk=32768, compressor=0.03, steps=8), call="step", timer=B.KERNEL_WORKER,
                                   bytes=lambda w: w.n * (12 * w.d + w.d // 4) + 4 * w.d),
        "k_topk_worker_two_pass": dict(setup=dict(chunk=32768, compressor=0.1, steps=1), call="step", timer=B.KERNEL_WORKER,
                                       bytes=lambda w: w.n * (12 * w.d + w.d // 4) + 4 * w.d),
        "k_topk_server_dense": dict(setup=dict(chunk=32768, compressor=0.03, steps=8), call="step", timer=B.KERNEL_SERVER,
                                    bytes=lambda w: w.n * (w.d // 8 + int(0.12 * w.d)) + 24 * w.d + w.d // 8),
        "k_error_norm_tiles": dict(setup=dict(chunk=32768), call="error_norms", timer=None,
                                   bytes=lambda w: 4 * (w.n + 1) * w.d),
    }


def _operator_cases():
    """Kernels of the operators beside the step: name -> function making (call, algorithmic bytes of the whole call)."""
    import torch

    from . import operators as O

    def tensor(rows, width, dtype=torch.bfloat16):
        return torch.empty(rows, width, device="cuda", dtype=dtype).normal_()

    def gradients(clip, big=8, in_place=False):
        sizes = [4 << 20] * big + [1 << 20] * 32 + [1024] * 64                   # big = 8: 67 M elements
        grads = [torch.empty(n, device="cuda").normal_() for n in sizes]
        tensors, d = O.TensorList(grads), sum(sizes)
        flat = torch.empty(d, device="cuda")
        if in_place:
            calls = itertools.count()
            return lambda: tensors.clip_grads(grads, 1e3 * 0.99 ** next(calls)), 8 * d       # each limit below the norm that the last one left
        if clip:
            return lambda: tensors.clip_grads(grads, 1.0, out=flat), 8 * d
        return lambda: tensors.grad_norm(grads), 4 * d

    def forward(rows, width, dtype=torch.bfloat16, group=None, stream=None):
        stream = stream or dtype
        x, r, w = tensor(rows, width, dtype), tensor(rows, width, stream), tensor(1, width, dtype)[0]
        nbytes = rows * width * (dtype.itemsize + 2 * stream.itemsize + (dtype.itemsize if group is None else 1))
        if group is None:
            return lambda: O.rms_norm_forward(x, w, r), nbytes
        return lambda: O.rms_norm_fp8(x, w, r, group=group), nbytes

    def backward(rows, width, dtype=torch.bfloat16, stream=None):
        both = stream is not None                                                # dx in both types
        stream = stream or dtype
        dy, h, dh, w = tensor(rows, width, dtype), tensor(rows, width, stream), tensor(rows, width, stream), tensor(1, width, dtype)[0]
        rstd = torch.rand(rows, device="cuda")
        return lambda: O.rms_norm_backward(dy, h, w, rstd, dh), rows * width * (2 * dtype.itemsize + (3 if both else 2) * stream.itemsize)

    def lookup(tokens, width, back=False, vocabulary=30_522):
        t = torch.randint(0, vocabulary, (tokens,), device="cuda")
        if back:
            dout, out = tensor(tokens, width), torch.empty(vocabulary, width, device="cuda")
            return lambda: O.embedding_backward(dout, t, vocabulary, out=out), 8 * tokens + 2 * tokens * width + 4 * vocabulary * width
        table = tensor(vocabulary, width)
        return lambda: O.embedding_forward(t, table, 2.0), 8 * tokens + 2 * width * (len(t.unique()) + tokens)

    def drop(rows, width, junction=True, pad=0):
        x, rng = tensor(rows, width + pad)[:, :width], torch.tensor([1, 2], device="cuda")
        r = tensor(rows, width) if junction else None
        return lambda: O.dropout_forward(x, 0.1, rng, 0, r), rows * width * (6 if junction else 4)

    def scan(batch, steps, width, back=False, dtype=torch.bfloat16):
        x, gate, dh = (torch.empty(batch, steps, width, device="cuda", dtype=dtype).normal_() for _ in range(3))
        n = batch * steps * width * dtype.itemsize
        if not back:
            return lambda: O.gated_scan_forward(x, gate), 3 * n
        starts = O.gated_scan_forward(x, gate, keep=True)[2]
        return lambda: O.gated_scan_backward(dh, x, gate, starts), 5 * n

    return {
        "k_embed": lambda: lookup(65_536, 1024), "k_embed_few": lambda: lookup(512, 1024, back=True), "k_embed_sort": lambda: lookup(65_536, 1024, back=True),
        "k_embed_zeros": lambda: lookup(65_536, 1024, back=True), "k_embed_sums": lambda: lookup(65_536, 1024, back=True), "k_embed_joins": lambda: lookup(65_536, 1024, back=True),
        "k_dropout": lambda: drop(8192, 4096, junction=False), "k_dropout_junction": lambda: drop(8192, 4096), "k_dropout_any": lambda: drop(8191, 4095, pad=1),
        "k_scan": lambda: scan(16, 2048, 2048), "k_scan_f32": lambda: scan(8, 2048, 2048, dtype=torch.float32), "k_scan_odd": lambda: scan(16, 2048, 2047), "k_scan_parts": lambda: scan(1, 32_768, 1024),
        "k_scan_back": lambda: scan(16, 2048, 2048, back=True), "k_scan_back_f32": lambda: scan(8, 2048, 2048, back=True, dtype=torch.float32),
        "k_tile_squares": lambda: gradients(False), "k_list_norm": lambda: gradients(False), "k_one_norm": lambda: gradients(False, 4), "k_scale_tiles": lambda: gradients(True),
        "k_scale_tiles_in_place": lambda: gradients(True, in_place=True),
        "k_rms_staged": lambda: forward(8192, 4096), "k_rms_staged_row_scale": lambda: forward(8192, 4096, group=0),
        "k_rms_staged_column_scales": lambda: forward(8192, 4096, group=128), "k_rms_staged_f32": lambda: forward(8192, 4096, torch.float32),
        "k_rms_staged_f32_stream": lambda: forward(8192, 4096, stream=torch.float32), "k_rms_rows": lambda: forward(512, 65_544, torch.float32),
        "k_rms_narrow": lambda: forward(200_000, 128), "k_rms_shifted": lambda: forward(8192, 4095),
        "k_rms_back_team": lambda: backward(8192, 4096), "k_rms_back_team_shifted": lambda: backward(8192, 4095), "k_rms_back_team_f32": lambda: backward(8192, 4096, torch.float32),
        "k_rms_back_team_f32_stream": lambda: backward(8192, 4096, stream=torch.float32), "k_rms_back_team_wide": lambda: backward(4096, 16_384), "k_rms_back_rows": lambda: backward(512, 65_544, torch.float32),
        "k_rms_back_shares": lambda: backward(8192, 4096),
    }


def _run_operator(args, make) -> int:
    import torch

    call, nbytes = make()
    for _ in range(3):
        call()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    e0.record()
    for _ in range(args.launches):
        call()
    e1.record()
    torch.cuda.synchronize()
    ms = e0.elapsed_time(e1) / args.launches
    print(json.dumps({"kernel": args.kernel, "launches": args.launches, "algorithmic_bytes_per_call": nbytes, "ms_per_call": ms,
                      "timed": "events around the whole call", "algorithmic_gbs": nbytes / (ms * 1e-3) / 1e9}))
    return 0


def main(argv=None) -> int:
    ap = argparse.ArgumentParser()
    ap.add_argument("--kernel", required=True)
    ap.add_argument("--d", type=int, default=1 << 25)
    ap.add_argument("--n", type=int, default=8)
    ap.add_argument("--launches", type=int, default=3)
    args = ap.parse_args(argv)

    import torch

    from . import binding as B
    from . import workloads as wl

    cases, operators = _cases(args), _operator_cases()
    if args.kernel in operators:
        return _run_operator(args, operators[args.kernel])
    if args.kernel not in cases:
        print("unknown kernel; one of: " + " ".join(sorted(cases) + sorted(operators)), file=sys.stderr)
        return 2
    case = cases[args.kernel]
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    if case["setup"] is None:                                   # the entry point without a context
        w = wl.sliced(wl.config(3), args.d).with_(n=1, chunk=32768)
        z = torch.empty(w.d, dtype=torch.float32, device="cuda").normal_()
        bits = torch.empty((w.d + 31) // 32, dtype=torch.int32, device="cuda")
        scales = torch.empty(w.n_chunks, dtype=torch.float32, device="cuda")
        stream = torch.cuda.current_stream().cuda_stream
        call = lambda: B.apms_compress_noalloc(z.data_ptr(), w.d, w.chunk, bits.data_ptr(), scales.data_ptr(), stream)
        call()
        ctx = None
    else:
        ctx, w, grads = _setup(args.d, args.n, **case["setup"])
        kind = case.get("call")
        if case.get("phase") == "warmup":
            ctx.restore(2, B.PHASE_WARMUP)
            call = lambda: ctx.warmup_step(grads)
        elif kind == "step":
            call = lambda: ctx.compressed_step(grads)
        elif kind == "worker_phase":
            def call():
                ctx.worker_phase(grads)
                ctx.server_phase_rows([ctx.message_ptrs(i)[0] for i in range(w.n)],
                                      [ctx.message_ptrs(i)[1] for i in range(w.n)], 0, ctx.C)
                ctx.apply_phase()
        elif kind == "first_worker_phase":
            def call():                                          # the binary32 momentum is authoritative again after set_state(M)
                ctx.set_state(B.STATE_M, ctx.get_state(B.STATE_M))
                ctx.compressed_step(grads)
        elif kind == "make_den":
            def call():                                          # a new v invalidates the stored sqrt(v) + eps
                ctx.set_state(B.STATE_V, ctx.get_state(B.STATE_V))
                ctx.compressed_step(grads)
        elif kind == "uncompressed":
            call = lambda: ctx.uncompressed_step(grads)
        elif kind == "error_norms":
            call = lambda: ctx.error_norms()
        else:
            raise AssertionError(kind)
        call()
    torch.cuda.synchronize()
    if ctx is not None and case["timer"] is not None:
        ctx.set_timing(True)
        ctx.kernel_time(case["timer"])
    e0.record()
    for _ in range(args.launches):
        call()
    e1.record()
    torch.cuda.synchronize()
    out = {"kernel": args.kernel, "d": w.d, "n": w.n, "chunk": w.chunk, "launches": args.launches,
           "algorithmic_bytes_per_launch": int(case["bytes"](w))}
    if ctx is not None and case["timer"] is not None:
        ms, cnt = ctx.kernel_time(case["timer"])
        out["ms_per_launch"] = ms / max(cnt, 1)
        out["timed"] = "library events around the kernel (and, for the worker, its finalize kernel)"
    else:
        out["ms_per_launch"] = e0.elapsed_time(e1) / args.launches
        out["timed"] = "events around the whole call"
    out["algorithmic_gbs"] = out["algorithmic_bytes_per_launch"] / (out["ms_per_launch"] * 1e-3) / 1e9
    print(json.dumps(out))
    return 0


if __name__ == "__main__":
    sys.exit(main())
