"""The operators beside the step, as far as they go without a GPU: what the C entry points refuse before anything is launched,
workspace sizes, and that there is no CPU path."""
import ctypes as C

import pytest
import torch

from paper_2008_11343_b200 import binding as B
from paper_2008_11343_b200 import build as libbuild
from paper_2008_11343_b200 import operators as O


@pytest.fixture(scope="module", autouse=True)
def lib():
    libbuild.build()
    return B.load()


def refused(call, words, status=B.ERR_INVALID_ARG):
    with pytest.raises(B.ApmsError) as e:
        call()
    assert e.value.status == status and words in str(e.value), str(e.value)


def test_a_list_of_tensors_is_checked_when_it_is_made():
    refused(lambda: B.apms_tensors_create([], []), "count >= 1")
    refused(lambda: B.apms_tensors_create([4, -1], [0, 0]), "tensor 1")
    refused(lambda: B.apms_tensors_create([4, 4], [0, 3]), "tensor 1 has an unknown element type")
    refused(lambda: B.apms_tensors_create([12], [0], [5], [6]), "no rows of 5")
    refused(lambda: B.apms_tensors_create([12], [0], [6], [5]), "5 apart")
    lib = B.load()
    n = (C.c_int64 * 1)(4)
    t = (C.c_int * 1)(0)
    assert lib.apms_tensors_create(None, 1, n, t, None, None) == B.ERR_INVALID_ARG
    h = C.c_void_p()
    assert lib.apms_tensors_create(C.byref(h), 1, n, t, n, None) == B.ERR_INVALID_ARG       # cols without strides
    assert h.value is None


def test_a_list_without_workspace_runs_nothing():
    h = B.apms_tensors_create([8, 0, 100_000], [B.GRAD_F32, B.GRAD_BF16, B.GRAD_F16])
    need = B.apms_tensors_workspace_bytes(h)
    assert 0 < need < 1 << 20 and need % 256 == 0
    ptrs = (C.c_void_p * 3)(256, 0, 256)
    refused(lambda: B.apms_grad_norm(h, ptrs, 256, None, None), "no workspace", B.ERR_BAD_STATE)
    refused(lambda: B.apms_clip_grads(h, ptrs, 1.0, None, 0, 256, None), "no workspace", B.ERR_BAD_STATE)
    refused(lambda: B.apms_tensors_bind(h, 128, need, None), "256-byte aligned")
    refused(lambda: B.apms_tensors_bind(h, 256, need - 1, None), "smaller", B.ERR_OOM)
    refused(lambda: B.apms_tensors_bind(None, 256, need, None), "needs a list")
    B.apms_tensors_destroy(h)
    B.apms_tensors_destroy(None)
    assert B.apms_tensors_workspace_bytes(None) == 0


def forward_args(**changes):
    a = B.RmsNormArgs(rows=2, width=8, x=256, x_stride=8, x_type=B.GRAD_BF16, residual=512, residual_stride=8, residual_type=B.GRAD_BF16,
                      weight=1024, weight_type=B.GRAD_F32, eps=1e-6, h=2048, y=4096, rstd=8192)
    for k, v in changes.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("changes,words", [
    ({"rows": -1}, "rows"), ({"width": 0}, "width"), ({"width": (1 << 24) + 1}, "width"), ({"x_type": 7}, "type"),
    ({"residual_type": B.GRAD_F16}, "x's type or binary32"), ({"weight_type": B.GRAD_F16}, "x's type or binary32"),
    ({"eps": -1.0}, "eps"), ({"eps": float("nan")}, "eps"), ({"x": None}, "NULL"), ({"h": None}, "NULL"), ({"rstd": None}, "NULL"),
    ({"x_stride": 7}, "stride"), ({"residual_stride": 7}, "stride"), ({"x": 257}, "aligned"), ({"weight": 1026}, "aligned"),
    ({"scales": 256, "group": 64}, "group"), ({"scales": 258}, "aligned"),
])
def test_the_norm_refuses(changes, words):
    refused(lambda: B.apms_rms_norm(forward_args(**changes), None), words)


def test_the_norm_of_no_rows_is_nothing():
    B.apms_rms_norm(forward_args(rows=0, x=None), None)
    assert B.load().apms_rms_norm(None, None) == B.ERR_INVALID_ARG


def backward_args(**changes):
    a = B.RmsNormBackwardArgs(rows=2, width=8, dy=256, dy_stride=8, dy_type=B.GRAD_BF16, h=512, h_stride=8, h_type=B.GRAD_F32, weight=1024,
                              weight_type=B.GRAD_BF16, rstd=2048, dh=4096, dh_stride=8, dx=8192, dresidual=16384, dweight=32768,
                              workspace_dev=65536, workspace_bytes=1 << 20)
    for k, v in changes.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("changes,words", [
    ({"rows": -1}, "rows"), ({"width": 0}, "width"), ({"dy_type": -1}, "type"), ({"h_type": B.GRAD_F16}, "dy's type or binary32"),
    ({"weight_type": B.GRAD_F16}, "dy's type or binary32"), ({"dweight": None}, "NULL"), ({"dx": None}, "NULL"), ({"dy": None}, "NULL"),
    ({"dy_stride": 7}, "stride"), ({"dh_stride": 7}, "stride"), ({"dresidual": 16386}, "aligned"), ({"dy": 257}, "aligned"),
])
def test_the_backward_pass_refuses(changes, words):
    refused(lambda: B.apms_rms_norm_backward(backward_args(**changes), None), words)


def test_the_backward_pass_needs_its_workspace():
    need = B.apms_rms_norm_backward_workspace_bytes(2, 8)
    assert need >= 8 * 4 and B.apms_rms_norm_backward_workspace_bytes(-1, 8) == 0 == B.apms_rms_norm_backward_workspace_bytes(2, 0)
    for bad in ({"workspace_dev": None}, {"workspace_dev": 65544}, {"workspace_bytes": need - 1}):
        refused(lambda: B.apms_rms_norm_backward(backward_args(**bad), None), "workspace", B.ERR_OOM)


def test_there_is_no_cpu_path():
    x, w = torch.ones(2, 8), torch.ones(8)
    for call in (lambda: O.rms_norm_forward(x, w), lambda: O.rms_norm_fp8(x, w), lambda: O.rms_norm_backward(x, x, w, torch.ones(2)),
                 lambda: O.TensorList([x]), lambda: O.TensorList([])):
        with pytest.raises(ValueError):
            call()


def test_rows_of_a_tensor():
    t, rows_of = torch.empty(6, 10), O._load().row_layout
    assert rows_of(t) == (60, 60) and rows_of(t[:, 2:7]) == (5, 10) and rows_of(t[::2, :4]) == (4, 20)
    assert rows_of(torch.empty(0, 3)) == (1, 1) and rows_of(torch.empty(2, 3, 8)[:, :, :5]) == (5, 8)
    for bad in (t.t(), t[:, ::2], torch.empty(2, 3, 8)[:, :2, :5], torch.empty(1, 4).expand(3, 4)):
        with pytest.raises(ValueError):
            rows_of(bad)
