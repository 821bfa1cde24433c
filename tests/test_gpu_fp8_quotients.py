"""The 8-bit norm's numbers are the quotients of the norm in fp32 and its scale, rounded to
nearest even, and the scales those of its magnitudes, bit for bit: also at ties, where
quotients of bf16 products often lie. Divided here on the CPU."""

import math

import pytest

from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu


def _want(torch, y, group):
    n, d = y.shape
    parts = torch.nn.functional.pad(y, (0, -d % (group or d))).view(n, -1, group or d)
    scales = (parts.abs().amax(dim=2) / 448.0).clamp(min=2.0 ** -126)
    q = (parts / scales[:, :, None]).view(n, -1)[:, :d]
    return q.to(torch.float8_e4m3fn), scales


@pytest.mark.parametrize("tokens,dim", [(300, 100), (2500, 1600), (40, 1001), (30, 9000),
                                        (7, 40000)])
@pytest.mark.parametrize("group", [0, 32, 128])
def test_quotients(tokens, dim, group):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(dim)
    for xt, wt in ((torch.bfloat16, torch.bfloat16), (torch.bfloat16, None),
                   (torch.float32, torch.float32)):
        x = torch.randn(tokens, dim, generator=gen, device="cuda")
        x[:, 5] *= 20.0
        x[0, :9] = torch.tensor([0.0, -0.0, 1.0, -1.0, 0.5, 1.5, 2.5, -3.5, 7.0], device="cuda")
        w = None if wt is None else (
            1.0 + 0.2 * torch.randn(dim, generator=gen, device="cuda")).to(wt)
        x = x.to(xt)
        y = ops.rms_norm(x, w, out_dtype=torch.float32).cpu()
        q, scales = ops.rms_norm_fp8(x, w, group=group)
        want, want_scales = _want(torch, y, group)
        assert torch.equal(scales.cpu(), want_scales)
        assert torch.equal(q.cpu().view(torch.uint8), want.view(torch.uint8))


def test_every_tie():
    """Rows whose largest magnitude takes 448 and that hold every number half way between two
    of e4m3, and their neighbours in fp32."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    numbers = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    ties = (numbers[1:] + numbers[:-1]) / 2
    one = torch.cat([numbers, ties, torch.nextafter(ties, torch.tensor(math.inf)),
                     torch.nextafter(ties, torch.tensor(0.0))])
    row = torch.cat([one, -one, torch.tensor([448.0, -0.0])])
    x = torch.stack([row * s for s in (1.0, 3.0, 1e-3, 2.0 ** 40, 0.7, 2.0 ** -30)]).cuda()
    for w in (None, torch.full((x.shape[1],), 0.1, device="cuda")):
        y = ops.rms_norm(x, w, eps=0.0, out_dtype=torch.float32).cpu()
        q, scales = ops.rms_norm_fp8(x, w, eps=0.0)
        want, want_scales = _want(torch, y, 0)
        assert torch.equal(scales.cpu(), want_scales)
        assert torch.equal(q.cpu().view(torch.uint8), want.view(torch.uint8))
