"""A small language model with one token table for its input and its output, trained
with the package's optimizers and operators:

  lookup        ops.embedding: rows of the table's bf16 copy
  body          residual blocks over the mean of the last few tokens (torch, autograd),
                with ops.rms_norm and ops.rms_norm_grad on the residual stream
  loss          ops.linear_cross_entropy against the same table, without keeping logits
  gradients     ops.linear_cross_entropy_grad writes the table's gradient buffer and the
                hidden states' gradient; after the body's backward pass
                ops.embedding_grad adds the lookup's share to the same buffer
  clipping      ops.GradNorm keeps all gradients together to one norm
  step          Muon for the blocks' matrices, LAMB for the norms' weights and for the
                table, which writes the bf16 copy that the next lookup and loss read

The data are synthetic: each token follows the one before by a fixed random rule three
times out of four, and is random otherwise, so the loss can fall to about a third of
the logarithm of the vocabulary's size.

Run: python examples/tied_lm.py [--steps 100]
"""

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1904_00962_amd import LAMB, Muon, ops  # noqa: E402

CONTEXT = 4  # tokens whose mean a position sees
IGNORE = -100


def batch(rule, tokens, gen):
    """Token ids and the ids that follow them, [tokens] each; the last has no target."""
    vocab = len(rule)
    ids = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
    kept = torch.rand(tokens, generator=gen, device="cuda") < 0.75
    # runs of the rule, from each random token on
    at = torch.arange(tokens, device="cuda")
    begin = torch.cummax(torch.where(kept, 0, at), dim=0).values
    for _ in range(int((at - begin).max())):
        follow = rule[torch.roll(ids, 1)]
        ids = torch.where(kept & (at > 0), follow, ids)
    targets = torch.roll(ids, -1)
    targets[-1] = IGNORE
    return ids, targets


class Norm(torch.autograd.Function):
    """(norm, sum) of the residual stream and a block's output, the norm in ``dtype``."""

    @staticmethod
    def forward(ctx, stream, branch, weight, dtype):
        norm, total = ops.rms_norm(branch, weight, residual=stream, out_dtype=dtype)
        ctx.save_for_backward(total, weight)
        return norm, total

    @staticmethod
    def backward(ctx, grad_norm, grad_total):
        total, weight = ctx.saved_tensors
        grad, grad_weight = torch.empty_like(total), torch.empty_like(weight)
        ops.rms_norm_grad(total, weight, grad_norm.contiguous(), grad, grad_weight,
                          grad_sum=grad_total.contiguous())
        return grad, grad, grad_weight, None


class Body(torch.nn.Module):
    def __init__(self, dim, blocks):
        super().__init__()
        make = lambda r, c: torch.nn.Parameter(  # noqa: E731
            torch.randn(r, c, device="cuda") / math.sqrt(c))
        self.up = torch.nn.ParameterList([make(2 * dim, dim) for _ in range(blocks)])
        self.down = torch.nn.ParameterList([make(dim, 2 * dim) for _ in range(blocks)])
        self.norms = torch.nn.ParameterList(
            [torch.nn.Parameter(torch.ones(dim, device="cuda")) for _ in range(blocks + 1)])

    def forward(self, rows):
        stream = rows.float()
        past = sum(torch.roll(stream, k, 0) for k in range(1, CONTEXT)) / (CONTEXT - 1)
        branch = 0.1 * past
        for up, down, weight in zip(self.up, self.down, self.norms):
            n, stream = Norm.apply(stream, branch, weight, torch.float32)
            branch = torch.relu(n @ up.t()) @ down.t()
        return Norm.apply(stream, branch, self.norms[-1], torch.bfloat16)[0]


def train(steps=100, vocab=2000, dim=128, blocks=2, tokens=2048, seed=0, report=None):
    """The mean loss of each step."""
    torch.manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rule = torch.randperm(vocab, generator=gen, device="cuda")
    table = torch.randn(vocab, dim, generator=gen, device="cuda").mul_(0.02)
    grad_table = torch.zeros(vocab, dim, dtype=torch.bfloat16, device="cuda")
    body = Body(dim, blocks)
    matrices, weights = [*body.up, *body.down], list(body.norms)
    for p in body.parameters():
        p.grad = torch.zeros_like(p)  # persistent: the plans bind the buffers
    lamb = LAMB([table], [grad_table], lr=0.02, weight_decay=0.0, clamp=(0.1, 10.0))
    copy = lamb.attach_bf16_copies()[0].view(vocab, dim)
    copy.copy_(table)
    muon = Muon([p.data for p in matrices], [p.grad for p in matrices], lr=0.01, momentum=0.9)
    lamb_weights = LAMB([p.data for p in weights], [p.grad for p in weights], lr=0.002)
    clipper = ops.GradNorm([grad_table] + [p.grad for p in body.parameters()])
    grad_hidden = torch.empty(tokens, dim, dtype=torch.bfloat16, device="cuda")
    scale = math.sqrt(dim)
    losses = []
    for step in range(steps):
        ids, targets = batch(rule, tokens, gen)
        rows = ops.embedding(ids, copy, scale=scale).requires_grad_()
        hidden = body(rows)
        mean, _, lse = ops.linear_cross_entropy(hidden.detach(), copy, targets,
                                                ignore_index=IGNORE)
        ops.linear_cross_entropy_grad(hidden.detach(), copy, targets, lse, grad_hidden,
                                      grad_table, ignore_index=IGNORE)
        for p in body.parameters():
            p.grad.zero_()
        hidden.backward(grad_hidden)
        ops.embedding_grad(ids, rows.grad, grad_table, scale=scale, accumulate=True)
        clipper.clip(1.0)
        muon.step()
        lamb_weights.step()
        lamb.step()
        losses.append(mean)
        if report and (step % 10 == 0 or step + 1 == steps):
            report("step %4d  loss %.4f" % (step, float(mean)))
    return [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=100)
    a = ap.parse_args()
    train(a.steps, report=lambda line: print(line, flush=True))


if __name__ == "__main__":
    main()
