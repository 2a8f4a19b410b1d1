"""The operators beside the compressed step, on torch CUDA tensors (the C calls: include/apms.h).

  TensorList       a model's gradients, many tensors: their norm, clipping in place, clipping INTO the flat gradient that
                   binding.Context's step functions take
  rms_norm         root-mean-square norm at a residual junction, differentiable
  rms_norm_forward, rms_norm_fp8, rms_norm_backward    its parts; 8-bit output (e4m3) with scales

Every call runs on torch's current stream and returns without a host synchronisation; there is no CPU path.
"""
from __future__ import annotations

from array import array
from typing import Optional, Sequence

import torch

from . import binding as B

_numel, _is_contiguous, _get_device, _data_ptr = (getattr(torch.Tensor, name) for name in ("numel", "is_contiguous", "get_device", "data_ptr"))
_TYPES = {torch.float32: B.GRAD_F32, torch.bfloat16: B.GRAD_BF16, torch.float16: B.GRAD_F16}


def _type(t, what: str) -> int:
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"{what} is {t.dtype}: float32, bfloat16 or float16 is needed")
    return kind


# ------------------------------------------------------------------------------------------ many tensors

class TensorList:
    """The sizes, types and layouts of a list of CUDA tensors of one device, and the memory its calls work in.

    Built once for a model's gradients; each call is given the tensors again (their addresses may change between calls, their sizes,
    types and strides may not).  A tensor is contiguous, or rows of consecutive elements a fixed distance apart (a column
    slice of a matrix).  Calls on another stream than the list's last one wait for that one."""

    def __init__(self, tensors: Sequence[torch.Tensor]):
        tensors = list(tensors)
        if not tensors:
            raise ValueError("a TensorList needs at least one tensor")
        self.device = tensors[0].device
        if any(not t.is_cuda or t.device != self.device for t in tensors):
            raise ValueError("the tensors of a TensorList lie on one CUDA device")
        self._numel = [t.numel() for t in tensors]
        self._dtypes = [t.dtype for t in tensors]
        self._strides = None if all(t.is_contiguous() for t in tensors) else [(t.shape, t.stride()) for t in tensors]
        self.numel = sum(self._numel)
        rows = [_rows_of(t) for t in tensors]
        self._h = None
        self._h = B.apms_tensors_create(self._numel, [_type(t, "a tensor") for t in tensors],
                                        [c for c, _ in rows], [s for _, s in rows])
        self._stream = torch.cuda.current_stream(self.device)
        nbytes = B.apms_tensors_workspace_bytes(self._h)
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            B.apms_tensors_bind(self._h, self.workspace.data_ptr(), nbytes, self._stream.cuda_stream)

    def __del__(self):
        if getattr(self, "_h", None):
            B.apms_tensors_destroy(self._h)
            self._h = None

    def grad_norm(self, tensors: Sequence[torch.Tensor]):
        """(||g||_2 over all tensors, the norm of each): float32, a scalar and len(tensors) values."""
        ptrs = self._addresses(tensors)
        out = torch.empty(1 + len(self._numel), dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            B.apms_grad_norm(self._h, ptrs, out.data_ptr(), out.data_ptr() + 4, self._enter())
        return out[0], out[1:]

    def clip_grads(self, tensors: Sequence[torch.Tensor], max_norm: float, out: Optional[torch.Tensor] = None):
        """Multiplies every element by min(1, max_norm / norm) and returns the norm before clipping (a float32 scalar).
        Without `out` in place; with it the tensors stay as they are and the clipped elements are written to `out`, one
        after the other: a flat gradient of self.numel elements for Context.warmup_step / compressed_step."""
        ptrs = self._addresses(tensors)
        flat, kind = None, B.GRAD_F32
        if out is not None:
            if not out.is_cuda or out.device != self.device or not out.is_contiguous() or out.numel() != self.numel:
                raise ValueError(f"out must be {self.numel} contiguous elements on {self.device}")
            flat, kind = out.data_ptr(), _type(out, "out")
            if self.numel == 0:
                flat = self.workspace.data_ptr()              # nothing is written; an empty tensor has no address
        norm = torch.empty((), dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            B.apms_clip_grads(self._h, ptrs, max_norm, flat, kind, norm.data_ptr(), self._enter())
        return norm

    def _addresses(self, tensors) -> array:
        """The tensors' addresses, once they are found to be laid out as the list's are."""
        if list(map(_numel, tensors)) != self._numel or [t.dtype for t in tensors] != self._dtypes:
            raise ValueError("the tensors differ from the list's in number, size or type")
        if self._strides is None:
            if not all(map(_is_contiguous, tensors)):
                raise ValueError("a tensor is not contiguous, as it was when the list was made")
        elif [(t.shape, t.stride()) for t in tensors] != self._strides:
            raise ValueError("the tensors' strides differ from the list's")
        if set(map(_get_device, tensors)) != {self.device.index}:
            raise ValueError(f"a tensor does not lie on {self.device}, as the list does")
        return array("Q", map(_data_ptr, tensors))

    def _enter(self) -> int:
        stream = torch.cuda.current_stream(self.device)
        if stream != self._stream:
            stream.wait_stream(self._stream)
            self.workspace.record_stream(stream)
            self._stream = stream
        return stream.cuda_stream


def _rows_of(t):
    """(elements of a row, distance between rows) of a tensor that is contiguous or rows of consecutive elements."""
    if t.is_contiguous():
        return max(1, t.numel()), max(1, t.numel())
    try:
        m = t.view(-1, t.shape[-1])
    except RuntimeError:
        m = None
    if m is None or m.stride(1) != 1 or m.stride(0) < m.shape[1]:
        raise ValueError(f"a tensor of shape {tuple(t.shape)} and strides {t.stride()} is no rows of consecutive elements; use .contiguous()")
    return m.shape[1], m.stride(0)


# ------------------------------------------------------------------------------------------ RMS norm

def _as_rows(t, what: str, width: int, device, rows: Optional[int] = None):
    """t as [rows, width] with consecutive elements in a row (copied only where its strides cannot be read that way)."""
    if t.device != device:
        raise ValueError(f"{what} lies on {t.device}, not on {device}")
    if t.dim() == 0 or t.shape[-1] != width or (rows is not None and t.numel() != rows * width):
        raise ValueError(f"{what} of shape {tuple(t.shape)} does not fit rows of width {width}")
    if t.is_contiguous():
        return t, width
    m = t.reshape(-1, width)
    if m.stride(1) != 1 or (m.shape[0] > 1 and m.stride(0) < width):
        m = m.contiguous()
    return m, m.stride(0)


def _weight(weight, width: int, device, narrow):
    if weight.device != device or weight.shape != (width,) or not weight.is_contiguous() or weight.dtype not in (narrow, torch.float32):
        raise ValueError(f"weight must be {width} contiguous elements on {device}, of {narrow} or float32")


def _forward(x, weight, residual, eps, group):
    if not x.is_cuda:
        raise ValueError("x must be a CUDA tensor; there is no CPU path")
    if x.dim() == 0 or x.shape[-1] == 0:
        raise ValueError(f"x of shape {tuple(x.shape)} has no rows of at least one element")
    a = B.RmsNormArgs()
    width = a.width = x.shape[-1]
    rows = a.rows = x.numel() // width
    a.x_type = _type(x, "x")
    _weight(weight, width, x.device, x.dtype)
    xr, a.x_stride = _as_rows(x, "x", width, x.device)
    a.x, a.weight, a.weight_type, a.eps = xr.data_ptr(), weight.data_ptr(), _TYPES[weight.dtype], eps
    h = x
    if residual is not None:
        if residual.shape != x.shape or residual.dtype not in (x.dtype, torch.float32):
            raise ValueError(f"residual must have x's shape, and its type or float32: {tuple(residual.shape)}, {residual.dtype}")
        rr, a.residual_stride = _as_rows(residual, "residual", width, x.device)
        h = torch.empty(x.shape, dtype=residual.dtype, device=x.device)
        a.residual, a.residual_type, a.h = rr.data_ptr(), _TYPES[residual.dtype], h.data_ptr()
    rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    a.rstd = rstd.data_ptr()
    scales = None
    if group is None:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    else:
        y = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=x.device)
        scales = torch.empty(*x.shape[:-1], -(-width // (group or width)), dtype=torch.float32, device=x.device)
        a.scales, a.group = scales.data_ptr(), group
    a.y = y.data_ptr()
    if rows:
        with torch.cuda.device(x.device):
            B.apms_rms_norm(a, torch.cuda.current_stream(x.device).cuda_stream)
    return y, scales, h, rstd


def rms_norm_forward(x, weight, residual=None, eps: float = 1e-6):
    """(y, h, rstd): h = x + residual (x itself without one), rstd = 1 / sqrt(mean(h^2) + eps) over the last dimension,
    y = h * rstd * weight.  residual and weight have x's type or float32; y has x's, h the residual's."""
    y, _, h, rstd = _forward(x, weight, residual, eps, None)
    return y, h, rstd


def rms_norm_fp8(x, weight, residual=None, eps: float = 1e-6, group: int = 0):
    """(q, scales, h, rstd): as rms_norm_forward, with y as float8_e4m3fn q and float32 scales, y ~ q * scale: one scale a row
    (group 0) or per 128 consecutive columns (group 128; the last group may be shorter)."""
    if group not in (0, 128):
        raise ValueError(f"group must be 0 (a scale per row) or 128, got {group}")
    return _forward(x, weight, residual, eps, group)


def rms_norm_backward(dy, h, weight, rstd, dh=None):
    """(dx, dweight) from what rms_norm_forward returned and the gradients dy of y and dh of h (None: zero); dx is the gradient of x
    and of the residual.  Where h's type is not dy's (a float32 residual stream) a third value is dx in h's type."""
    if not dy.is_cuda:
        raise ValueError("dy must be a CUDA tensor; there is no CPU path")
    if dy.dim() == 0 or dy.shape[-1] == 0:
        raise ValueError(f"dy of shape {tuple(dy.shape)} has no rows of at least one element")
    a = B.RmsNormBackwardArgs()
    width = a.width = dy.shape[-1]
    rows = a.rows = dy.numel() // width
    a.dy_type = _type(dy, "dy")
    if h.dtype not in (dy.dtype, torch.float32):
        raise ValueError(f"h must have dy's type or float32, not {h.dtype}")
    _weight(weight, width, dy.device, dy.dtype)
    if rstd.dtype != torch.float32 or rstd.numel() != rows or not rstd.is_contiguous() or rstd.device != dy.device:
        raise ValueError(f"rstd must be {rows} contiguous float32 values on {dy.device}")
    dyr, a.dy_stride = _as_rows(dy, "dy", width, dy.device)
    hr, a.h_stride = _as_rows(h, "h", width, dy.device, rows)
    a.dy, a.h, a.h_type, a.weight, a.weight_type, a.rstd = dyr.data_ptr(), hr.data_ptr(), _TYPES[h.dtype], weight.data_ptr(), _TYPES[weight.dtype], rstd.data_ptr()
    if dh is not None:
        if dh.dtype != h.dtype:
            raise ValueError(f"dh must have h's type {h.dtype}, not {dh.dtype}")
        dhr, a.dh_stride = _as_rows(dh, "dh", width, dy.device, rows)
        a.dh = dhr.data_ptr()
    dx = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
    dresidual = None if h.dtype == dy.dtype else torch.empty(dy.shape, dtype=h.dtype, device=dy.device)
    dweight = torch.empty_like(weight)
    nbytes = B.apms_rms_norm_backward_workspace_bytes(rows, width)
    workspace = torch.empty(nbytes, dtype=torch.uint8, device=dy.device)
    a.dx, a.dweight, a.workspace_dev, a.workspace_bytes = dx.data_ptr(), dweight.data_ptr(), workspace.data_ptr(), nbytes
    if dresidual is not None:
        a.dresidual = dresidual.data_ptr()
    with torch.cuda.device(dy.device):
        B.apms_rms_norm_backward(a, torch.cuda.current_stream(dy.device).cuda_stream)
    return (dx, dweight) if dresidual is None else (dx, dweight, dresidual)


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
        dx, dweight, *dresidual = rms_norm_backward(dy, h, weight, rstd, dh)
        return dx, dweight, (dresidual[0] if dresidual else dx) if ctx.junction else None, None


def rms_norm(x, weight, residual=None, eps: float = 1e-6):
    """y = rms_norm(x, weight), or (y, h) = rms_norm(x, weight, residual) with h = x + residual; differentiable in all three."""
    return _RmsNorm.apply(x, weight, residual, eps)
