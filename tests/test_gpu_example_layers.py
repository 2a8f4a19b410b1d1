"""The example with sequences and dropout: embedding, norms, recurrence, dropout, clipping into the flat gradients and the step together, and their gradients."""
import math
import os
import sys

import pytest
import torch
import torch.nn.functional as F

import layers_oracle as oracle

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from paper_2008_11343_b200 import binding as B


@pytest.mark.parametrize("eight_bit", [False, True])
def test_it_runs(eight_bit):
    import train_block

    losses, norms, phase, launches = train_block.train(steps=6, warmup=4, batch=128, sequence=32, dropout=0.1, eight_bit=eight_bit)
    assert all(math.isfinite(v) for v in losses + norms) and phase == B.PHASE_COMPRESSED and launches >= 6


def plain_loss(leaves, tokens, targets, dropout, seed, step):
    """loss_of in 64 bits, from its definition."""
    embedding, *blocks, last_norm, head = leaves

    def norm(h, weight):
        return h * (h.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * weight

    out, stream, site = embedding[tokens], 0.0, 0
    while blocks:
        for recurrence in (True, False):
            weight, w_in, w_out, *blocks = blocks
            stream = stream + out
            y = norm(stream, weight) @ w_in
            if recurrence:
                x, gate = y.chunk(2, dim=-1)
                h, states = torch.zeros_like(x[:, 0]), []
                for t in range(x.shape[1]):
                    z = torch.sigmoid(-gate[:, t])
                    h = h + z * (x[:, t] - h)
                    states.append(h)
                out = torch.stack(states, 1) @ w_out
            else:
                out = F.gelu(y) @ w_out
            kept, scale = oracle.kept(out.numel(), dropout, seed, step, site)
            out = out * kept.view(out.shape).to(out.device) * scale
            site += 1
    return F.cross_entropy((norm(stream + out, last_norm) @ head).flatten(0, -2), targets.flatten())


def test_its_gradients():
    """binary32 leaves.  Each of the about 30 products, norms and recurrences on a path rounds sums of up to 128 terms: 30 * 128 * 2^-24 = 2.3e-4 of a gradient's size."""
    import train_block

    gen = torch.Generator(device="cuda").manual_seed(3)
    vocab, width = 60, 64
    leaves = [torch.ones(s, device="cuda") if len(s) == 1 else torch.empty(s, device="cuda").normal_(0.0, s[0] ** -0.5, generator=gen) for s in train_block.shapes(vocab, width, 2, recurrent=True)]
    leaves = [p.requires_grad_() for p in leaves]
    wide = [p.detach().double().requires_grad_() for p in leaves]
    tokens = torch.randint(vocab, (5, 37), device="cuda", generator=gen)
    targets = torch.randint(vocab, (5, 37), device="cuda", generator=gen)
    loss = train_block.loss_of(leaves, tokens, targets, dropout=0.2, rng=torch.tensor([11, 5], device="cuda"))
    want = plain_loss(wide, tokens, targets, 0.2, 11, 5)
    assert abs(float(loss.detach()) - float(want.detach())) < 2.3e-4 * float(want.detach())
    for got, expected in zip(torch.autograd.grad(loss, leaves), torch.autograd.grad(want, wide)):
        assert float((got.double() - expected).norm()) < 2.3e-4 * float(expected.norm())
