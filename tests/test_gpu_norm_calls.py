"""Calls of the norm and of gradient plans that their documentation allows beside the usual
ones: a sum that is not kept, gradients of the weight alone and added to what was there, and
long lists in a captured graph."""

import math

import pytest

import rms_reference as R
from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu

EPS = 1e-6


@pytest.mark.parametrize("dim", [40, 1600, 1601, 9000, 40000])
@pytest.mark.parametrize("tokens", [1, 50, 3000])
def test_a_sum_that_is_not_kept(tokens, dim):
    torch = torch_cuda()
    from paper_1904_00962_amd import _ops, ops
    gen = torch.Generator(device="cuda").manual_seed(dim)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    bf16, f32 = _ops.LAMB_DTYPE_BF16, _ops.LAMB_DTYPE_F32
    x, res, w = rand(tokens, dim).bfloat16(), rand(tokens, dim), rand(dim)
    want, _ = ops.rms_norm(x, w, residual=res, eps=EPS)
    q, scales, _ = ops.rms_norm_fp8(x, w, residual=res, eps=EPS, group=64)
    kept = res.clone()
    r = _ops.lamb_rms(x.data_ptr(), res.data_ptr(), w.data_ptr(), dim, dim, tokens, dim, bf16, f32,
                      f32, EPS)
    out, q2, scales2 = torch.empty_like(x), torch.empty_like(q), torch.empty_like(scales)
    stream = torch.cuda.current_stream().cuda_stream
    _ops.lamb_rms_forward(r, None, 0, out.data_ptr(), dim, bf16, stream)
    _ops.lamb_rms_quantize(r, None, 0, q2.data_ptr(), dim, scales2.data_ptr(), 64, stream)
    assert torch.equal(out, want) and torch.equal(res, kept)
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(scales2, scales)


# one workgroup, several, and two passes
@pytest.mark.parametrize("tokens,dim", [(3, 64), (5, 4097), (1000, 250), (2000, 1600), (700, 8192),
                                        (10, 9000), (300, 20001)])
@pytest.mark.parametrize("dwt", ["float32", "bfloat16"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_the_weight_alone(tokens, dim, dwt, accumulate):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(dim)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, dy, w = rand(tokens, dim).bfloat16(), rand(tokens, dim), rand(dim)
    old = (10.0 * rand(dim)).to(getattr(torch, dwt))
    got = []
    for grad_x in (None, torch.empty_like(x)):
        gw = old.clone()
        ops.rms_norm_grad(x, w, dy, grad_x, gw, eps=EPS, accumulate=accumulate)
        R.check_grads(grad_x, gw, x, w, dy, None, EPS, old if accumulate else None)
        got.append(gw)
    assert torch.equal(*got)
    # the gradient of x alone is the same as with the weight's
    alone = torch.empty_like(x)
    ops.rms_norm_grad(x, w, dy, alone, eps=EPS, accumulate=accumulate)
    assert torch.equal(alone, grad_x)


@pytest.mark.parametrize("kind", ["l2", "linf"])
def test_long_lists_in_a_graph(kind):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(5)
    grads = [torch.empty(n, device="cuda", dtype=t) for n, t in (
        (5_000_001, torch.float32), (0, torch.float32), (3_000_003, torch.bfloat16),
        (17, torch.float32), (2_000_000, torch.bfloat16))]
    outputs = [torch.empty(g.numel(), dtype=torch.bfloat16, device="cuda") for g in grads]
    plan = ops.GradNorm(grads, outputs, norm=kind)
    fill = lambda: [g.copy_(torch.randn(g.numel(), generator=gen, device="cuda"))  # noqa: E731
                    for g in grads]
    fill(), plan.clip(1.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.clip(1.0)
    results = (*outputs, plan.norms, plan.total, plan.found_nonfinite)
    for k in range(4):
        fill()
        if k == 2:
            grads[0][123456] = math.inf
        graph.replay()
        torch.cuda.synchronize()
        held = [t.clone() for t in results]
        for t in results:
            t.zero_()
        plan.clip(1.0)
        torch.cuda.synchronize()
        for a, b in zip(held, results):
            assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)), k
        assert int(plan.found_nonfinite) == (k == 2)
