"""The norm's paths that only calls of many rows take: teams of half the lanes forward, and
backward many rows to a workgroup, whose terms of the weight's gradient are summed in
parts."""

import pytest

import rms_reference as R
from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu

EPS = 1e-6


def _rows(torch, gen, tokens, dim, dtype, sigma=1.0):
    t = torch.randn(tokens, dim, generator=gen, device="cuda")
    t *= torch.exp(2 * torch.rand(tokens, 1, generator=gen, device="cuda")) * sigma
    t[:, :: max(1, dim // 3)] *= 12.0
    return t.to(dtype)


# From 2048 rows on, widths up to 7/8 of a team's columns; 2051 rows leave a last workgroup
# of several teams unfilled.
@pytest.mark.parametrize("dim", [520, 896, 1032, 1600, 1792, 2056, 3584, 4104, 7168])
@pytest.mark.parametrize("tokens", [2047, 2048, 2051])
def test_half_the_lanes(tokens, dim):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(dim + tokens)
    w = (1.0 + 0.3 * torch.randn(dim, generator=gen, device="cuda"))
    for xt, rt, wt in ((torch.bfloat16, None, torch.bfloat16), (torch.float32, None, None),
                       (torch.bfloat16, torch.bfloat16, torch.float32),
                       (torch.bfloat16, torch.float32, torch.float32),
                       (torch.float32, torch.float32, None)):
        x = _rows(torch, gen, tokens, dim, xt)
        res = None if rt is None else _rows(torch, gen, tokens, dim, rt, 3.0)
        weight = None if wt is None else w.to(wt)
        h = x if res is None else (x.float() + res.float()).to(rt)
        got = ops.rms_norm(x, weight, residual=res, eps=EPS)
        if res is not None:
            got, summed = got
            assert torch.equal(summed, h)
        R.check_norm(got, h, weight, EPS)
        for group in (0, 32, 64, 128, 256):
            q, scales, *summed = ops.rms_norm_fp8(x, weight, residual=res, eps=EPS, group=group)
            if res is not None:
                assert torch.equal(summed[0], h)
            R.check_fp8(q, scales, h, weight, EPS, group)


@pytest.mark.parametrize("tokens,dim,xt,yt", [
    (700_001, 40, "bfloat16", "bfloat16"), (300_003, 250, "bfloat16", "float32"),
    (100_001, 500, "float32", "bfloat16"), (40_001, 1024, "bfloat16", "bfloat16"),
    (32_768, 1600, "float32", "bfloat16"), (20_003, 4096, "bfloat16", "bfloat16"),
    (10_001, 8192, "bfloat16", "bfloat16"), (10_003, 7001, "bfloat16", "bfloat16"),
    (4_001, 9000, "bfloat16", "bfloat16")])
def test_gradients(tokens, dim, xt, yt):
    """More than 32 turns to a workgroup's teams."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(dim)
    xt, yt = getattr(torch, xt), getattr(torch, yt)
    x, dy = _rows(torch, gen, tokens, dim, xt), _rows(torch, gen, tokens, dim, yt)
    ds = _rows(torch, gen, tokens, dim, xt)
    w = 1.0 + 0.3 * torch.randn(dim, generator=gen, device="cuda")
    gx, gw = torch.empty_like(x), torch.empty_like(w)
    ops.rms_norm_grad(x, w, dy, gx, gw, eps=EPS, grad_sum=ds)
    R.check_grads(gx, gw, x, w, dy, ds, EPS)
    again = torch.empty_like(gx), torch.empty_like(gw)
    ops.rms_norm_grad(x, w, dy, *again, eps=EPS, grad_sum=ds)
    assert torch.equal(again[0], gx) and torch.equal(again[1], gw)


@pytest.mark.parametrize("x,dy", [(0.9, 1.9), (1.3, 0.3), (1.1, 0.9)])
@pytest.mark.parametrize("tokens,dim,teams", [(1 << 23, 24, 16), (1 << 19, 1600, 1)])
def test_like_terms(tokens, dim, teams, x, dy):
    """Rows alike, so that all terms of a sum are one number, and 512 turns or more to a team.
    Of a sum of n like terms the roundings, each half a step of what is summed so far at most,
    are (n + 1) / 2 half steps of the whole: 32 terms to a sum, at most as many of those as
    512 workgroups leave to one, then the workgroup's teams; a term has two roundings and the
    result one. One chain of 512 such terms in fp32 is 72 half steps off and more."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    rows = torch.full((tokens, dim), x, device="cuda")
    grads = torch.full((tokens, dim), dy, device="cuda")
    gw = torch.empty(dim, device="cuda")
    ops.rms_norm_grad(rows, None, grads, None, gw, eps=EPS)
    one = torch.tensor([x, dy, EPS], dtype=torch.float32).double()
    want = float(tokens * one[1] * one[0] / torch.sqrt(one[0] ** 2 + one[2]))
    sums = tokens / (512 * teams * 32)
    steps = 2 + (32 + 1) / 2 + (sums + 1) / 2 + (teams + 1) / 2 + 1
    off = float((gw.double() - want).abs().max()) / want
    assert off <= steps * R.ULP, off / R.ULP
