"""Gradients of rows at the ends of fp32, whose 1 / rms no fp32 number holds to its
precision, or at all: the results are ordinary numbers where grad_out makes them so. The
bounds are those of rms_reference.py: a power of two taken out of 1 / rms rounds nothing."""

import pytest

import rms_reference as R
from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu

# a row's size, and that of its grad_out: 1 / rms is 4e-39 to 2e41
ROWS = [(3.3e38, 1e10), (1e38, 1e12), (1.2e-38, 1e-4), (1e-41, 1e-6), (1e-38, 0.0), (1e-41, 0.0),
        (2.0, 1.0), (3.0, 0.0), (1e-39, 1e-30), (3.3e38, 1e-3)]


@pytest.mark.parametrize("dim", [1, 6, 64, 100, 700, 1600, 8000, 8191, 9000, 9001])
@pytest.mark.parametrize("xt,gt", [("float32", "float32"), ("bfloat16", "bfloat16"),
                                   ("bfloat16", "float32")])
def test_gradients(dim, xt, gt):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    xt, gt = getattr(torch, xt), getattr(torch, gt)
    gen = torch.Generator(device="cuda").manual_seed(dim)
    # more rows than one workgroup takes, in two orders
    rows = ROWS * 5 + ROWS[::-1] * 4
    n = len(rows)
    size, grad = torch.tensor(rows, device="cuda", dtype=torch.float64).T[:, :, None]
    if xt == torch.bfloat16:
        size = size.clamp(min=4e-40)  # below 4.6e-41 they are 0
    signs = torch.where(torch.rand(n, dim, generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    x = (signs * size * (0.5 + 0.5 * torch.rand(n, dim, generator=gen, device="cuda"))).to(xt)
    assert bool((x != 0).all() & x.isfinite().all())
    w = torch.randn(dim, generator=gen, device="cuda")
    dy = (grad * torch.randn(n, dim, generator=gen, device="cuda")).float()
    for ds in (None, torch.randn(n, dim, generator=gen, device="cuda").to(gt)):
        for some in (slice(None), slice(0, 10), slice(3, 4)):
            part = None if ds is None else ds[some]
            gx, gw = torch.empty(n, dim, dtype=gt, device="cuda")[some], torch.empty_like(w)
            ops.rms_norm_grad(x[some], w, dy[some], gx, gw, eps=0.0, grad_sum=part)
            R.check_grads(gx, gw, x[some], w, dy[some], part, 0.0)
            zero = (grad[some, 0] == 0).nonzero()[:, 0]
            assert torch.equal(gx[zero], torch.zeros_like(gx[zero]) if ds is None else part[zero])
