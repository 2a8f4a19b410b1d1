"""Kernels of the layers' operators that only large calls take: several groups of eight a thread, one team of warps an SM over several rounds."""
import functools

import pytest
import torch

import layers_oracle as oracle
from paper_2008_11343_b200 import operators as O
from test_gpu_layers import BF16, F16, F32, KINDS, check_scan, gates, normal, rng_of, tokens_for

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("out", KINDS)
@pytest.mark.parametrize("count,width", [(5001, 1048), (9001, 1048), (150_001, 64)])
def test_lookup_of_many_rows(count, width, kind, out):
    """5.2, 9.4 and 9.6 million elements; the last CTA has fewer groups than its threads take."""
    tokens, weight = tokens_for(count, 3000, 1), normal((3000, width), kind, seed=2, pad=8)
    oracle.within(O.embedding_forward(tokens, weight, 7.3, dtype=out), *oracle.embedding(tokens, weight, 7.3))


@functools.lru_cache(maxsize=1)
def mask(rows, width):
    kept, scale = oracle.kept(rows * width, 0.3, 77, 8, 9)
    return kept.view(rows, width).cuda(), scale


def dropped(x, residual=None):
    kept, scale = mask(*x.shape)
    v = torch.where(kept, x.double() * scale, 0.0)
    if residual is None:
        return v, v.abs() * 2.01 * oracle.U32
    h = v + residual.double()
    return h, v.abs() * 2.01 * oracle.U32 + h.abs() * oracle.U32


@pytest.mark.parametrize("kind,stream", [(F32, None), (BF16, None), (F16, None), (F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("pad", [(0, 0), (8, 0), (0, 16), (24, 8)])
def test_dropout_of_many_rows(kind, stream, pad):
    """9.3 million elements, in one run and in rows that are apart."""
    rows, width = 9001, 1032
    x = normal((rows, width), kind, seed=3, pad=pad[0])
    residual = None if stream is None else normal((rows, width), stream, 2.0, seed=4, pad=pad[1])
    h, used = O.dropout_forward(x, 0.3, rng_of(77, 8), 9, residual)
    oracle.within(h, *dropped(x, residual))
    dh = normal((rows, width), stream or kind, seed=5, pad=pad[1])
    oracle.within(O.dropout_backward(dh, 0.3, used, 9, dtype=kind), *dropped(dh))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("batch,width", [(150, 64), (160, 70), (149, 33), (80, 196), (75, 203)])
def test_scan_of_more_slabs_than_sms(kind, batch, width):
    """Over four rounds, with rows on 16 bytes, on 4 and (16 bits) on 2."""
    shape = (batch, 203, width)
    x, gate, dh = normal(shape, kind, seed=6), gates(shape, kind, 7), normal(shape, kind, seed=8)
    check_scan(x, gate, normal((batch, width), seed=9), dh, normal((batch, width), seed=10))


@pytest.mark.parametrize("kind", KINDS)
def test_scan_of_halves_of_rows_of_more_slabs_than_sms(kind):
    both, dh = normal((16, 300, 2 * 1280), kind, seed=11), normal((16, 300, 1280), kind, seed=12)
    x, gate = both[..., :1280], both[..., 1280:]
    check_scan(x, gate, None, dh)
