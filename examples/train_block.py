"""A small pre-norm residual network trained with the compressed step, every worker's gradients clipped on their way in.

    python examples/train_block.py [--steps 60] [--workers 4] [--eight-bit] [--sequence 32] [--dropout 0.1]

What runs of the package, per step: for every worker the forward pass - the tokens' rows (operators.embedding), the RMS norm at each
residual junction (operators.rms_norm; with --eight-bit the matrix products read what the norm's 8-bit output stands for), with
--sequence a gated linear recurrence over the positions in front of each block (operators.gated_scan), with --dropout dropout behind each of them
(operators.dropout: one pair of numbers a worker, advanced once a step, the place in the network as the site) - and its backward pass, the
worker's gradients - bfloat16 matrices, binary32 norm weights - clipped by their global norm INTO that worker's flat binary32
gradient (operators.TensorList.clip_grads), and one step of Algorithm 1 on the flat gradients (Context.step: Adam during
warmup, the 1-bit compressed step after it).  The task is synthetic: the next token is a fixed affine map of the
current one, with --sequence of the one before it (nothing is asked of a sequence's first one).
"""
from __future__ import annotations

import argparse
import math
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch
import torch.nn.functional as F

from paper_2008_11343_b200 import binding as B
from paper_2008_11343_b200 import operators


class _EightBitNorm(torch.autograd.Function):
    """operators.rms_norm whose y went through its 8-bit form; the gradient passes the rounding unchanged."""

    @staticmethod
    def forward(ctx, x, weight, stream):
        q, scales, h, rstd = operators.rms_norm_fp8(x, weight, stream)
        ctx.save_for_backward(h, weight, rstd)
        return (q.float() * scales).to(x.dtype), h

    @staticmethod
    def backward(ctx, dy, dh):
        if torch.is_grad_enabled():                                       # create_graph=True: nothing to differentiate again
            raise RuntimeError("no second derivatives through the 8-bit norm")
        dx, dweight, dstream = operators.rms_norm_backward(dy.contiguous(), *ctx.saved_tensors, dh)
        return dx, dweight, dstream


def shapes(vocab: int, width: int, layers: int, recurrent: bool = False):
    """Parameter shapes in the flat vector's order."""
    block = [(width,), (width, 2 * width), (2 * width, width)]            # norm weight, in, out
    if recurrent:
        block = [(width,), (width, 2 * width), (width, width), *block]    # norm weight, values and gates, out
    return [(vocab, width), *(block * layers), (width,), (width, vocab)]


def labels(tokens, vocab: int):
    """What is to be predicted at each token; -100: nothing, which the loss leaves out."""
    if tokens.dim() == 1:
        return (tokens * 5 + 3) % vocab
    return F.pad((tokens[:, :-1] * 5 + 3) % vocab, (1, 0), value=-100)


def loss_of(leaves, tokens, targets, eight_bit: bool = False, dropout: float = 0.0, rng=None):
    """Activations of the matrices' type on a binary32 residual stream.  Tokens of two dimensions are sequences: every block begins with a recurrence."""
    embedding, *blocks, last_norm, head = leaves
    norm = _EightBitNorm.apply if eight_bit else operators.rms_norm
    recurrent, site = tokens.dim() == 2, 0
    out = operators.embedding(tokens, embedding)
    stream = torch.zeros(out.shape, dtype=torch.float32, device=out.device)
    while blocks:
        for sublayer in ("recurrence", "mlp") if recurrent else ("mlp",):
            weight, w_in, w_out, *blocks = blocks
            y, stream = norm(out, weight, stream)
            if sublayer == "mlp":
                out = F.gelu(y @ w_in) @ w_out
            else:
                x, gate = (y @ w_in).chunk(2, dim=-1)
                out = operators.gated_scan(x, gate)[0] @ w_out
            if dropout:
                out = operators.dropout(out, dropout, rng, site)
                site += 1
    y, _ = norm(out, last_norm, stream)
    return F.cross_entropy((y @ head).float().flatten(0, -2), targets.flatten())


def train(steps: int = 60, workers: int = 4, vocab: int = 256, width: int = 192, layers: int = 3, batch: int = 512,
          warmup: int = 40, lr: float = 5e-3, max_norm: float = 1.0, eight_bit: bool = False, seed: int = 0, sequence: int = 0,
          dropout: float = 0.0):
    """Mean loss over the workers and mean gradient norm before clipping, one of each per step.  sequence: 0, or a divisor of batch above 1."""
    if sequence and (sequence < 2 or batch % sequence):
        raise ValueError(f"sequence must be 0 or a divisor of the batch of {batch} tokens above 1, not {sequence}")
    gen = torch.Generator(device="cuda").manual_seed(seed)
    sizes = shapes(vocab, width, layers, recurrent=sequence > 0)
    counts = [math.prod(s) for s in sizes]
    d = sum(counts)
    flat = torch.cat([torch.ones(n, device="cuda") if len(s) == 1 else torch.empty(n, device="cuda").normal_(0.0, s[0] ** -0.5 if s[0] != vocab else 1.0, generator=gen)
                      for n, s in zip(counts, sizes)])
    ctx = B.Context(d, workers, 0.9, 0.999, 1e-8, lr, chunk=4096)
    ctx.set_params(flat)
    ctx.set_schedule(B.Schedule(warmup_steps=warmup, peak_lr=lr, lr_ramp_steps=5, lr_decay=0.7, lr_decay_every=10))
    flat_grads = [torch.empty(d, device="cuda") for _ in range(workers)]
    rngs = [torch.tensor([seed + i, 0], device="cuda") for i in range(workers)]            # dropout's seed and step, of each worker
    gradients, losses, norms = None, [], []
    for _ in range(steps):
        leaves = [v.view(s) if len(s) == 1 else v.view(s).bfloat16() for v, s in zip(flat.split(counts), sizes)]
        leaves = [p.detach().requires_grad_() for p in leaves]
        step_losses, step_norms = [], []
        for i in range(workers):
            tokens = torch.randint(vocab, (batch // sequence, sequence) if sequence else (batch,), device="cuda", generator=gen)
            loss = loss_of(leaves, tokens, labels(tokens, vocab), eight_bit, dropout, rngs[i])
            rngs[i][1] += 1
            grads = torch.autograd.grad(loss, leaves)
            if gradients is None:
                gradients = operators.TensorList(grads)
            step_norms.append(gradients.clip_grads(grads, max_norm, out=flat_grads[i]))
            step_losses.append(loss.detach())
        ctx.step(flat_grads)
        ctx.get_params(out=flat)
        losses.append(torch.stack(step_losses).mean())
        norms.append(torch.stack(step_norms).mean())
    phase, launches = ctx.phase, ctx.launch_count
    ctx.close()
    return [float(v) for v in losses], [float(v) for v in norms], phase, launches


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--eight-bit", action="store_true", help="the norms' 8-bit output feeds the matrix products")
    ap.add_argument("--sequence", type=int, default=0, help="tokens come as sequences of this length (a divisor of 512 above 1), with a recurrence in front of each block")
    ap.add_argument("--dropout", type=float, default=0.0)
    args = ap.parse_args()
    losses, norms, phase, launches = train(steps=args.steps, workers=args.workers, eight_bit=args.eight_bit, sequence=args.sequence, dropout=args.dropout)
    for k in range(0, len(losses), 10):
        print(f"step {k:4d}  loss {losses[k]:.4f}  gradient norm {norms[k]:.3f}")
    print(f"step {len(losses) - 1:4d}  loss {losses[-1]:.4f}  ({'compressed' if phase == B.PHASE_COMPRESSED else 'warmup'} phase, {launches} step kernels)")


if __name__ == "__main__":
    main()
