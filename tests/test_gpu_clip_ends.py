"""Clipping by factors that fp32 does not hold to its precision, or at all: gradients at the
end of fp32's range, whose norm lies past it, and scales past it. The products are then those
of 64 bits, each rounded to fp32 once and to bf16 from there."""

import math

import pytest

from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu

SIZES = [40000, 1, 0, 16385, 2047, 7]


def _case(torch, size, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    grads = []
    for n in SIZES:
        g = (torch.rand(n + 1, generator=gen, device="cuda") * size).to(dtype)[1:]
        grads.append(torch.where(torch.rand(n, generator=gen, device="cuda") < 0.1, 0.0, g))
    return grads


# norm, size of the gradients, limit, scale
CASES = [("l1", 3e38, 1.0, 1.0),         # f = 1 / 1e43
         ("l2", 3e38, 2.0, -1.0),        # 1 / 2e40
         ("linf", 3e38, 1.0, 1.0),       # 1 / 3e38: a subnormal fp32 number
         ("l1", 3e38, 1e-6, 3e-5),       # 1e-49: no fp32 number at all
         ("l2", 1e-20, math.inf, 1e40), ("l2", 1e-38, 1e30, -1e70), ("l2", 0.0, 1.0, 1e300),
         ("l2", 1e30, math.inf, 1e-42), ("linf", 1e-30, 1e9, 3.4028236e38)]


@pytest.mark.parametrize("kind,size,limit,scale", CASES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("out", [None, "float32", "bfloat16"])
def test_clip(kind, size, limit, scale, dtype, out):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    grads = _case(torch, size, getattr(torch, dtype), len(CASES))
    before = [g.clone() for g in grads]
    outputs = None if out is None else [
        torch.full((g.numel(),), math.nan, dtype=getattr(torch, out), device="cuda")
        for g in grads]
    plan = ops.GradNorm(grads, outputs, norm=kind)
    total = float(plan.clip(limit, scale=scale))
    assert math.isfinite(total)
    f = math.copysign(limit / total, scale) if abs(scale) * total > limit else scale
    factor = torch.tensor(f, dtype=torch.float64, device="cuda")
    for g, o in zip(before, plan.outputs):
        want = (g.double() * factor).float()
        assert bool(want.isfinite().all())
        assert torch.equal(o, want.to(o.dtype))
    assert int(plan.found_nonfinite) == 0
