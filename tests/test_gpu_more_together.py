"""The operators of a training step together, as the example calls them: lookup, norms of
the residual stream, loss, their gradients, the gradients' norm and clipping, and steps,
against the same model in torch's autograd in 64 bits.

The looked-up rows and the hidden states are bf16 in both (a block's relu has no derivative
at 0, so a rounding that only one of them had would decide entries there). Tolerance, as
2-norms: the gradients of the hidden states and of the rows are rounded to bf16 (2^-8 of each
entry at most, less in the mean), the softmax too (2.5e-3), and the table's gradient twice:
five roundings of up to 2^-8, 2e-2 together; everything else is fp32 (the blocks' products
are torch's, 1e-6). Clipping has the factor's rounding and the products' (2^-8 for the bf16
table)."""

import importlib.util
import math
import os

import pytest

import ops_reference
from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "tied_lm.py")


def _example():
    spec = importlib.util.spec_from_file_location("tied_lm", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


def _plain(torch, example, body, table, ids, targets, scale):
    """(mean loss, gradients of the table, the matrices and the norms' weights) in fp64."""
    table = table.double().requires_grad_()
    params = [p.detach().double().requires_grad_() for p in body.parameters()]
    n = len(body.up)
    up, down, weights = params[:n], params[n:2 * n], params[2 * n:]

    def norm(x, w):
        return x * torch.rsqrt(x.square().mean(dim=1, keepdim=True) + 1e-6) * w

    def rounded(x):
        return x + (x.detach().float().bfloat16().double() - x.detach())

    x = rounded(table[ids] * scale)
    x = x + 0.1 * sum(torch.roll(x, k, 0) for k in range(1, example.CONTEXT)) / (
        example.CONTEXT - 1)
    for u, d, w in zip(up, down, weights):
        x = x + torch.relu(norm(x, w) @ u.t()) @ d.t()
    logits = rounded(norm(x, weights[-1])) @ table.t()
    keep = targets != example.IGNORE
    loss = (torch.logsumexp(logits[keep], dim=1)
            - logits[keep].gather(1, targets[keep][:, None])[:, 0]).mean()
    return loss.detach(), torch.autograd.grad(loss, [table] + params)


@pytest.mark.parametrize("tokens,dim,vocab,blocks", [(130, 64, 300, 2), (77, 60, 91, 1)])
def test_a_step_against_autograd(tokens, dim, vocab, blocks):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    example = _example()
    torch.manual_seed(3)
    gen = torch.Generator(device="cuda").manual_seed(3)
    ids, targets = example.batch(torch.randperm(vocab, generator=gen, device="cuda"), tokens, gen)
    body = example.Body(dim, blocks)
    with torch.no_grad():
        for w in body.norms:
            w += 0.2 * torch.randn(dim, generator=gen, device="cuda")
    copy = torch.randn(vocab, dim, generator=gen, device="cuda").mul_(0.1).bfloat16()
    scale = math.sqrt(dim)
    loss, want = _plain(torch, example, body, copy, ids, targets, scale)
    grad_table = torch.empty_like(copy)
    rows = ops.embedding(ids, copy, scale=scale).requires_grad_()
    hidden = body(rows)
    mean, _, lse = ops.linear_cross_entropy(hidden.detach(), copy, targets)
    grad_hidden = torch.empty_like(hidden)
    ops.linear_cross_entropy_grad(hidden.detach(), copy, targets, lse, grad_hidden, grad_table)
    hidden.backward(grad_hidden)
    ops.embedding_grad(ids, rows.grad, grad_table, scale=scale, accumulate=True)
    got = [grad_table] + [p.grad for p in body.parameters()]
    assert abs(float(mean) - float(loss)) <= 2e-2 * float(loss)
    for k, (a, b) in enumerate(zip(got, want)):
        assert ops_reference.relative(a, b) < 2e-2, k
    # clipped together
    total = torch.stack([g.square().sum() for g in want]).sum().sqrt()
    before = [g.double() for g in got]
    clipper = ops.GradNorm(got)
    seen = float(clipper.clip(0.5 * float(total)))
    assert abs(seen / float(total) - 1.0) <= 2e-2
    for a, b in zip(got, before):
        assert ops_reference.relative(a, b * (0.5 * float(total) / seen)) <= 2.0 ** -8


def test_the_example_runs():
    torch_cuda()
    losses = _example().train(steps=8, vocab=300, dim=40, tokens=256)
    assert len(losses) == 8 and all(math.isfinite(v) for v in losses)
    assert abs(losses[0] - math.log(300)) < 0.5
