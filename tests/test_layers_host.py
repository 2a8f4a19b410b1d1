"""The layers' operators as far as they go without a GPU: what is refused before anything is launched, workspace sizes, the generator against its published
values, and derivatives of derivatives."""
import pytest
import torch

import layers_oracle as oracle
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


def changed(a, changes):
    for k, v in changes.items():
        setattr(a, k, v)
    return a


def lookup(**changes):
    return changed(B.EmbeddingArgs(count=3, vocab=5, width=8, tokens=256, token_bytes=8, weight=512, weight_stride=8, weight_type=B.GRAD_BF16, scale=1.0, out=1024,
                                   out_type=B.GRAD_F32), changes)


@pytest.mark.parametrize("changes,words", [
    ({"count": -1}, "count"), ({"count": 1 << 31}, "count"), ({"vocab": 0}, "vocab"), ({"vocab": 1 << 31}, "vocab"), ({"width": 0}, "width"), ({"width": (1 << 19) + 1}, "width"),
    ({"count": (1 << 31) - 1, "width": 1 << 19}, "2^40"), ({"token_bytes": 2}, "4 or 8"), ({"weight_type": 3}, "type"), ({"out_type": -1}, "type"), ({"tokens": None}, "NULL"),
    ({"weight": None}, "NULL"), ({"out": None}, "NULL"), ({"weight_stride": 7}, "stride"), ({"tokens": 260}, "aligned"), ({"weight": 513}, "aligned"), ({"out": 1026}, "aligned"),
])
def test_the_lookup_refuses(changes, words):
    refused(lambda: B.apms_embedding(lookup(**changes), None), words)


def gradient(**changes):
    return changed(B.EmbeddingBackwardArgs(count=3, vocab=5, width=8, tokens=256, token_bytes=4, dout=512, dout_stride=8, dout_type=B.GRAD_BF16, scale=1.0, dweight=1024,
                                           dweight_type=B.GRAD_F32, workspace_dev=4096, workspace_bytes=1 << 20), changes)


@pytest.mark.parametrize("changes,words", [
    ({"count": -1}, "count"), ({"vocab": 0}, "vocab"), ({"width": 0}, "width"), ({"token_bytes": 16}, "4 or 8"), ({"dout_type": 3}, "type"), ({"dweight_type": 9}, "type"),
    ({"dweight": None}, "NULL"), ({"tokens": None}, "NULL"), ({"dout": None}, "NULL"), ({"dout_stride": -8}, "stride"), ({"tokens": 258}, "aligned"), ({"dout": 513}, "aligned"),
    ({"dweight": 1026}, "aligned"),
])
def test_the_gradient_refuses(changes, words):
    refused(lambda: B.apms_embedding_backward(gradient(**changes), None), words)


def test_the_gradient_needs_its_workspace():
    need = B.apms_embedding_backward_workspace_bytes(3000, 5, 8)
    assert need >= 2 * 3000 * 8 and 0 == B.apms_embedding_backward_workspace_bytes(-1, 5, 8) == B.apms_embedding_backward_workspace_bytes(3000, 0, 8) == B.apms_embedding_backward_workspace_bytes(1024, 5, 8)
    for bad in ({"workspace_dev": None}, {"workspace_dev": 4096 + 128}, {"workspace_bytes": need - 1}):
        refused(lambda: B.apms_embedding_backward(gradient(count=3000, **bad), None), "workspace", B.ERR_OOM)


def drop(**changes):
    return changed(B.DropoutArgs(rows=2, width=8, x=256, x_stride=8, x_type=B.GRAD_BF16, residual=512, residual_stride=8, p=0.1, rng_dev=1024, site=0, h=2048, h_type=B.GRAD_BF16,
                                 used_dev=4096), changes)


@pytest.mark.parametrize("changes,words", [
    ({"rows": -1}, "rows"), ({"width": 0}, "width"), ({"rows": 1 << 20, "width": (1 << 14) + 1}, "2^34"), ({"rows": 1 << 62, "width": 8}, "2^34"), ({"x_type": 3}, "type"), ({"h_type": 3}, "type"),
    ({"h_type": B.GRAD_F16}, "binary32 with a residual"), ({"residual": None, "h_type": B.GRAD_F32}, "binary32 x without one"), ({"p": -0.1}, "p must"), ({"p": 1.1}, "p must"), ({"p": float("nan")}, "p must"),
    ({"site": -1}, "site"), ({"site": 1 << 32}, "site"), ({"rng_dev": None}, "rng_dev"), ({"rng_dev": 1028}, "8-byte"), ({"used_dev": 4100}, "8-byte"), ({"x": None}, "NULL"), ({"h": None}, "NULL"),
    ({"x_stride": -8}, "stride"), ({"residual_stride": -8}, "stride"), ({"x": 257}, "aligned"), ({"h": 2049}, "aligned"), ({"residual": 513}, "aligned"),
])
def test_dropout_refuses(changes, words):
    refused(lambda: B.apms_dropout(drop(**changes), None), words)


def scan(**changes):
    return changed(B.GatedScanArgs(batch=2, steps=3, width=8, x=256, x_batch_stride=24, x_step_stride=8, gate=512, gate_batch_stride=24, gate_step_stride=8, type=B.GRAD_BF16, state=None,
                                   h=1024, last=2048, starts=None), changes)


def scan_back(**changes):
    return changed(B.GatedScanBackwardArgs(batch=2, steps=3, width=8, dh=4096, dh_batch_stride=24, dh_step_stride=8, x=256, x_batch_stride=24, x_step_stride=8, gate=512, gate_batch_stride=24,
                                           gate_step_stride=8, type=B.GRAD_BF16, starts=8192, dlast=None, dx=16384, dgate=32768, dstate=65536), changes)


SIZES = [({"batch": -1}, "below 0"), ({"steps": -1}, "below 0"), ({"width": 0}, "width"), ({"batch": 1 << 16, "width": 1 << 16}, "2^31"), ({"batch": 1 << 16, "width": 1 << 15, "steps": 1 << 10}, "2^40"),
         ({"type": 5}, "type"), ({"x": None}, "NULL"), ({"gate": None}, "NULL"), ({"x_step_stride": -1}, "stride"), ({"gate_batch_stride": -1}, "stride"), ({"x": 257}, "aligned")]


@pytest.mark.parametrize("changes,words", SIZES + [({"h": None}, "NULL"), ({"last": None}, "NULL"), ({"state": 130}, "aligned"), ({"last": 2050}, "aligned"), ({"starts": 8}, "aligned"), ({"h": 1025}, "aligned")])
def test_the_scan_refuses(changes, words):
    refused(lambda: B.apms_gated_scan(scan(**changes), None), words)


@pytest.mark.parametrize("changes,words", SIZES + [({"dh": None}, "NULL"), ({"starts": None}, "NULL"), ({"dx": None}, "NULL"), ({"dgate": None}, "NULL"), ({"dh_step_stride": -1}, "stride"),
                                                   ({"dstate": 65538}, "aligned"), ({"dlast": 2}, "aligned"), ({"dgate": 32769}, "aligned")])
def test_the_scan_backward_refuses(changes, words):
    refused(lambda: B.apms_gated_scan_backward(scan_back(**changes), None), words)


@pytest.mark.parametrize("changes,words", [({"batch": -1}, "below 0"), ({"width": 0}, "width"), ({"type": 3}, "type"), ({"x": None}, "NULL"), ({"state": None}, "NULL"), ({"next": None}, "NULL"),
                                           ({"h": None}, "NULL"), ({"x_stride": -1}, "stride"), ({"gate": 513}, "aligned"), ({"next": 1026}, "aligned")])
def test_the_step_refuses(changes, words):
    a = B.GatedScanStepArgs(batch=2, width=8, x=256, x_stride=8, gate=512, gate_stride=8, type=B.GRAD_BF16, state=1024, next=1024, h=2048)
    refused(lambda: B.apms_gated_scan_step(changed(a, changes), None), words)


def test_long_sequences_of_few_channels_need_a_workspace():
    need = B.apms_gated_scan_workspace_bytes(1, 5000, 64, B.GRAD_BF16)
    assert need > 0 == B.apms_gated_scan_workspace_bytes(1, 5000, 64, 7) == B.apms_gated_scan_workspace_bytes(1, 100, 64, B.GRAD_BF16) == B.apms_gated_scan_workspace_bytes(-1, 5000, 64, 0)
    long = dict(batch=1, steps=5000, width=64, x_step_stride=64, gate_step_stride=64)
    for bad in ({}, {"workspace_dev": 4096 + 8, "workspace_bytes": need}, {"workspace_dev": 4096, "workspace_bytes": need - 1}):
        refused(lambda: B.apms_gated_scan(scan(**long, **bad), None), "workspace", B.ERR_OOM)
        refused(lambda: B.apms_gated_scan_backward(scan_back(**long, dh_step_stride=64, **bad), None), "workspace", B.ERR_OOM)


def test_without_arguments_or_work():
    lib = B.load()
    for call in (lib.apms_embedding, lib.apms_embedding_backward, lib.apms_dropout, lib.apms_gated_scan, lib.apms_gated_scan_backward, lib.apms_gated_scan_step):
        assert call(None, None) == B.ERR_INVALID_ARG
    B.apms_embedding(lookup(count=0, tokens=None, out=None), None)
    B.apms_dropout(drop(rows=0, x=None, h=None, used_dev=None), None)
    B.apms_gated_scan(scan(batch=0, x=None, h=None, last=None), None)
    B.apms_gated_scan_backward(scan_back(batch=0, dh=None), None)
    assert B.apms_gated_scan_starts_bytes(2, 0, 8) == 0 == B.apms_gated_scan_starts_bytes(-1, 3, 8)
    assert B.apms_gated_scan_starts_bytes(2, 3, 8) % (2 * 4) == 0 < B.apms_gated_scan_starts_bytes(2, 3, 8)


def test_there_is_no_cpu_path():
    x, w, t, rng = torch.ones(2, 3, 8), torch.ones(5, 8), torch.ones(2, 3, dtype=torch.int64), torch.zeros(2, dtype=torch.int64)
    state = torch.ones(2, 8)
    for call in (lambda: O.embedding(t, w), lambda: O.embedding_backward(x, t, 5), lambda: O.dropout(x, 0.1, rng), lambda: O.dropout_backward(x, 0.1, rng), lambda: O.gated_scan(x, x),
                 lambda: O.gated_scan_backward(x, x, x, x), lambda: O.gated_scan_step(state, state, state)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_the_generator_gives_its_published_values():
    """The known answers published with the method, for 10 and for 7 rounds."""
    def words(counter, key, rounds):
        return [int(w[0]) for w in oracle.philox([[c] for c in counter], key, rounds)]
    top = 0xFFFFFFFF
    assert words([0] * 4, [0] * 2, 10) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert words([top] * 4, [top] * 2, 10) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert words([0] * 4, [0] * 2, 7) == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]


def test_second_derivatives_are_refused_not_dropped(monkeypatch):
    """With stand-ins for the kernels, on the CPU."""
    plain = lambda x, gate: x.detach() * gate.detach()
    monkeypatch.setattr(O, "gated_scan_forward", lambda x, gate, state=None, keep=False: (plain(x, gate), x.detach()[:, -1], x.detach()))
    monkeypatch.setattr(O, "gated_scan_backward", lambda dh, x, gate, starts, dlast=None: (dh * gate, dh * x, dh[:, 0].detach()))
    monkeypatch.setattr(O, "embedding_forward", lambda t, w, scale=1.0, dtype=None: w.detach()[t] * scale)
    monkeypatch.setattr(O, "embedding_backward", lambda d, t, n, scale, dtype: torch.zeros(n, d.shape[-1], dtype=d.dtype).index_add_(0, t.flatten(), d.detach().flatten(0, -2)) * scale)
    monkeypatch.setattr(O, "dropout_forward", lambda x, p, rng, site=0, residual=None: (x.detach() + residual.detach(), rng))
    monkeypatch.setattr(O, "dropout_backward", lambda dh, p, used, site, dtype: dh.detach())
    x, gate, w, r = (torch.randn(*s, dtype=torch.float64).requires_grad_() for s in ((2, 3, 4), (2, 3, 4), (5, 4), (2, 3, 4)))
    t, rng = torch.tensor([[1, 0, 2], [4, 4, 1]]), torch.zeros(2, dtype=torch.int64)
    for out, leaf in ((O.gated_scan(x, gate)[0], x), (O.embedding(t, w, 2.0), w), (O.dropout(x, 0.5, rng, 0, r), x)):
        first, = torch.autograd.grad(out.square().sum(), leaf, retain_graph=True)
        again, = torch.autograd.grad(out.square().sum(), leaf, create_graph=True)
        assert torch.equal(first, again) and not first.requires_grad
        with pytest.raises(RuntimeError, match="second derivative"):
            again.sum().backward()
