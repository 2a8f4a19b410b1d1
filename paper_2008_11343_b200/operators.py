"""The operators beside the compressed step, on torch CUDA tensors (the C calls: include/apms.h; checks, outputs and calls:
csrc/torch_operators.cpp).

  TensorList       a model's gradients, many tensors: their norm, clipping in place, clipping INTO the flat gradient that
                   binding.Context's step functions take
  rms_norm         root-mean-square norm at a residual junction, differentiable
  rms_norm_forward, rms_norm_fp8, rms_norm_backward    its parts; 8-bit output (e4m3) with scales
  embedding        lookup of scaled rows, differentiable; embedding_forward, embedding_backward (into the flat gradient's place)
  dropout          at a residual junction, its mask never stored, differentiable; dropout_forward, dropout_backward
  gated_scan       the gated linear recurrence over sequences, differentiable; gated_scan_forward, gated_scan_backward, and
                   gated_scan_step for one token

Every call runs on torch's current stream and returns without a host synchronisation; there is no CPU path.  Arguments that do not
fit raise ValueError, what the library refuses raises binding.ApmsError.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

from . import binding as B

_ext = None


def _load():
    """The extension (_operators.so, built by build.py), with the entry points of the library that binding has loaded."""
    global _ext
    if _ext is None:
        lib = B.load()
        if not os.path.exists(os.path.join(B.HERE, "_operators.so")):
            raise ImportError("_operators.so is not built; run `python -m paper_2008_11343_b200.build` (there is no fallback path)")
        from . import _operators

        names = [n for n in B.SIGNATURES if n.startswith(("apms_tensors_", "apms_grad_", "apms_clip_", "apms_rms_", "apms_embedding", "apms_dropout", "apms_gated_"))] + ["apms_last_error"]
        _operators.bind(B.ApmsError, {n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in names})
        _ext = _operators
    return _ext


class TensorList:
    """The sizes, types and layouts of a list of CUDA tensors of one device, and the memory its calls work in.

    Built once for a model's gradients; each call is given the tensors again (their addresses may change between calls, their
    sizes, types and strides may not).  A tensor is dense - contiguous, or with its elements in another order (transposed, channels
    last) - or rows of consecutive elements a fixed distance apart (a column slice of a matrix).  `numel` is the total of elements.

    Calls on another stream than the list's last one wait for that one.  Calls may be captured by torch.cuda.graph on any stream: each
    works in memory of the graph's pool, so replays need no order among the list's other calls; they read the list's tables, so the list
    has to live as long as the graph.  The list itself is built outside a capture."""

    def __init__(self, tensors: Sequence[torch.Tensor]):
        self._list, self.numel = _load().list_create(tensors)

    def grad_norm(self, tensors: Sequence[torch.Tensor]):
        """(||g||_2 over all tensors, the norm of each): float32, a scalar and len(tensors) values."""
        return _ext.grad_norm(self._list, tensors)

    def clip_grads(self, tensors: Sequence[torch.Tensor], max_norm: float, out: Optional[torch.Tensor] = None):
        """Multiplies every element by min(1, max_norm / norm) and returns the norm before clipping (a float32 scalar).
        Without `out` in place; with it the tensors stay as they are and the clipped elements are written to `out`, one
        after the other, each tensor's in the order of their indexes (one whose memory has another order is copied on the way): a flat
        gradient of self.numel elements for Context.warmup_step / compressed_step."""
        return _ext.clip_grads(self._list, tensors, max_norm, out)


def rms_norm_forward(x, weight, residual=None, eps: float = 1e-6):
    """(y, h, rstd): h = x + residual (x itself without one), rstd = 1 / sqrt(mean(h^2) + eps) over the last dimension,
    y = h * rstd * weight.  residual and weight have x's type or float32; y has x's, h the residual's."""
    return _load().rms_norm(x, weight, residual, eps, -1)


def rms_norm_fp8(x, weight, residual=None, eps: float = 1e-6, group: int = 0):
    """(q, scales, h, rstd): as rms_norm_forward, with y as float8_e4m3fn q and float32 scales, y ~ q * scale: one scale a row
    (group 0) or per 128 consecutive columns (group 128; the last group may be shorter)."""
    if group not in (0, 128):
        raise ValueError(f"group must be 0 (a scale per row) or 128, got {group}")
    return _load().rms_norm(x, weight, residual, eps, group)


def rms_norm_backward(dy, h, weight, rstd, dh=None):
    """(dx, dweight) from what rms_norm_forward returned and the gradients dy of y and dh of h (None: zero); dx is the gradient of x
    and of the residual.  Where h's type is not dy's (a float32 residual stream) a third value is dx in h's type."""
    return _load().rms_norm_backward(dy, h, weight, rstd, dh)


class _RmsNormGradient(torch.autograd.Function):
    """rms_norm_backward where a graph of the backward pass is being built (create_graph=True): the kernels leave nothing to
    differentiate, so its own backward pass raises.  (torch's once_differentiable would return constants where dy needs no gradient,
    though h and the weight do.)"""

    @staticmethod
    def forward(ctx, dy, h, weight, rstd, dh):
        return rms_norm_backward(dy, h, weight, rstd, dh)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("rms_norm has first derivatives only: its second derivatives are not implemented")


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        y, h, rstd = rms_norm_forward(x, weight, residual, eps)
        ctx.save_for_backward(h, weight, rstd)
        ctx.set_materialize_grads(False)
        ctx.x_type, ctx.junction = x.dtype, residual is not None
        return y if residual is None else (y, h)

    @staticmethod
    def backward(ctx, dy, dh=None):
        h, weight, rstd = ctx.saved_tensors
        if dy is None:                                       # only h was used: the norm contributes nothing
            return None if dh is None else dh.to(ctx.x_type), None, dh, None
        gradient = _RmsNormGradient.apply if torch.is_grad_enabled() else rms_norm_backward
        dx, dweight, *dresidual = gradient(dy, h, weight, rstd, dh)
        return dx, dweight, (dresidual[0] if dresidual else dx) if ctx.junction else None, None


def rms_norm(x, weight, residual=None, eps: float = 1e-6):
    """y = rms_norm(x, weight), or (y, h) = rms_norm(x, weight, residual) with h = x + residual; differentiable in all three,
    once: a second derivative raises RuntimeError."""
    return _RmsNorm.apply(x, weight, residual, eps)


class _FirstDerivative(torch.autograd.Function):
    """call(*args) where a graph of the backward pass is being built (create_graph=True): its own backward pass raises."""

    @staticmethod
    def forward(ctx, name, call, *args):
        ctx.name = name
        return call(*args)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError(f"{ctx.name} has first derivatives only: its second derivatives are not implemented")


def _derivative(name, call, *args):
    return _FirstDerivative.apply(name, call, *args) if torch.is_grad_enabled() else call(*args)


# ------------------------------------------------------------------------------------------ embedding

def embedding_forward(tokens, weight, scale: float = 1.0, dtype: Optional[torch.dtype] = None):
    """weight[tokens] * scale, in dtype (the weight's without one), of shape (*tokens.shape, width): formed in binary32, rounded once.  A token outside
    [0, len(weight)) gives zeros.  tokens: int64 or int32; weight: (vocabulary, width), float32, bfloat16 or float16."""
    return _load().embedding(tokens, weight, scale, dtype)


def embedding_backward(dout, tokens, vocabulary: int, scale: float = 1.0, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None):
    """The weight's gradient, (vocabulary, width): row v is scale times the sum of dout's rows at the tokens v, zeros where there are none.  Every
    row is written, once, in dtype (dout's without one), or to `out`: contiguous, such as the weight's place in a flat gradient."""
    return _load().embedding_backward(dout, tokens, vocabulary, scale, dtype, out)


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, weight, scale, dtype):
        ctx.save_for_backward(tokens)
        ctx.rows, ctx.scale, ctx.dtype = weight.shape[0], scale, weight.dtype
        return embedding_forward(tokens, weight, scale, dtype)

    @staticmethod
    def backward(ctx, dout):
        return None, _derivative("embedding", embedding_backward, dout, ctx.saved_tensors[0], ctx.rows, ctx.scale, ctx.dtype), None, None


def embedding(tokens, weight, scale: float = 1.0, dtype: Optional[torch.dtype] = None):
    """embedding_forward, differentiable in the weight (once: a second derivative raises RuntimeError)."""
    return _Embedding.apply(tokens, weight, scale, dtype)


# ------------------------------------------------------------------------------------------ dropout

def dropout_forward(x, p: float, rng, site: int = 0, residual=None):
    """(h, used): h = residual + x / (1 - p) where the mask keeps x and residual (0 without one) where it does not.  rng: two int64 numbers (seed, step)
    on x's device; the mask is a function of them, of `site` (which tells the calls of a step apart) and of the element's index alone.  They are read when
    the kernel runs: add 1 to rng[1] once per step, in a captured graph too.  used: a copy of them, for dropout_backward.  p counts in steps of
    2^-16, and 1 / (1 - p) is of the p so rounded.  residual: x's type or float32; h has the residual's type."""
    return _load().dropout(x, p, rng, site, residual, None, True)


def dropout_backward(dh, p: float, used, site: int = 0, dtype: Optional[torch.dtype] = None):
    """The gradient of dropout_forward's x from that of h (the residual's is dh): dh / (1 - p) where the mask kept x, else 0, in dtype (dh's without one;
    another than dh's from float32 only)."""
    return _load().dropout(dh, p, used, site, None, dtype, False)


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, rng, site, residual):
        h, used = dropout_forward(x, p, rng, site, residual)
        ctx.save_for_backward(used)
        ctx.p, ctx.site, ctx.dtype, ctx.junction = p, site, x.dtype, residual is not None
        return h

    @staticmethod
    def backward(ctx, dh):
        dx = _derivative("dropout", dropout_backward, dh, ctx.p, ctx.saved_tensors[0], ctx.site, ctx.dtype) if ctx.needs_input_grad[0] else None
        return dx, None, None, None, dh if ctx.junction else None


def dropout(x, p: float, rng, site: int = 0, residual=None):
    """dropout_forward's h, differentiable in x and residual (once: a second derivative in x raises RuntimeError)."""
    return _Dropout.apply(x, p, rng, site, residual)


# ------------------------------------------------------------------------------------------ gated linear recurrence

def gated_scan_forward(x, gate, state=None, keep: bool = False):
    """(h, last, starts): over the steps of x and gate, (batch, steps, width) of one type, h_t = h_(t-1) + sigmoid(-gate_t) (x_t - h_(t-1)) for every
    channel, from `state` ((batch, width) float32; zeros without one).  States are binary32 from step to step; h has x's type, last is the state
    behind the last step (float32).  starts: with keep what gated_scan_backward needs, else None.  A gate of +infinity keeps the state, one of -infinity
    replaces it by x (where a packed sequence begins, say) - as long as x and the state are finite: 0 times infinity is NaN."""
    return _load().gated_scan(x, gate, state, keep)


def gated_scan_backward(dh, x, gate, starts, dlast=None):
    """(dx, dgate, dstate) from the gradients dh of h and dlast (float32; None: zero) of last."""
    return _load().gated_scan_backward(dh, x, gate, starts, dlast)


def gated_scan_step(x, gate, state, out=None):
    """One token of every sequence: x and gate (batch, width); returns h and puts the new states into `out`, or into state itself."""
    return _load().gated_scan_step(x, gate, state, out)


class _GatedScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, state, recorded):
        keep = recorded and any(ctx.needs_input_grad)        # the latter are the inputs' own wishes, in every mode
        h, last, starts = gated_scan_forward(x, gate, state, keep)
        if keep:
            ctx.save_for_backward(x, gate, starts)
        ctx.set_materialize_grads(False)
        return h, last

    @staticmethod
    def backward(ctx, dh, dlast):
        x, gate, starts = ctx.saved_tensors
        if dh is None and dlast is None:
            return None, None, None, None
        if dh is None:
            dh = torch.zeros_like(x)
        dx, dgate, dstate = _derivative("gated_scan", gated_scan_backward, dh, x, gate, starts, dlast)
        return dx, dgate, dstate if ctx.needs_input_grad[2] else None, None


def gated_scan(x, gate, state=None):
    """(h, last) of gated_scan_forward, differentiable in all three (once: a second derivative raises RuntimeError)."""
    return _GatedScan.apply(x, gate, state, torch.is_grad_enabled())
