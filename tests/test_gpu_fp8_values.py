"""The 8-bit norm's numbers are the norm in fp32 times its scale's inverse, rounded to nearest
even, and the scales those of its magnitudes, bit for bit: also at ties, where quotients of
bf16 products often lie. Computed here on the CPU; but at ties they are the quotients too."""

import math

import pytest

from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu


def _want(torch, y, group):
    n, d = y.shape
    parts = torch.nn.functional.pad(y, (0, -d % (group or d))).view(n, -1, group or d)
    scales = (parts.abs().amax(dim=2) / 448.0).clamp(min=2.0 ** -126)
    q = (parts * (1.0 / scales[:, :, None])).view(n, -1)[:, :d].to(torch.float8_e4m3fn)
    # where a quotient in 64 bits is more than 2^-23 of it from the middle of two numbers
    exact = (parts.double() / scales.double()[:, :, None]).view(n, -1)[:, :d]
    divided = exact.float().to(torch.float8_e4m3fn)
    other = (q.view(torch.uint8) != divided.view(torch.uint8)).nonzero(as_tuple=True)
    middle = (q.double()[other] + divided.double()[other]) / 2
    assert bool(((exact[other] - middle).abs() <= 2.0 ** -23 * middle.abs()).all())
    return q, scales


@pytest.mark.parametrize("tokens,dim", [(300, 100), (2500, 1600), (40, 1001), (30, 9000),
                                        (7, 40000)])
@pytest.mark.parametrize("group", [0, 32, 128])
def test_values(tokens, dim, group):
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


@pytest.mark.parametrize("size", [1e-30, 1e-34, 1e-36, 1e-37, 1e-38, 1e-40, 1e-44, 1e34])
@pytest.mark.parametrize("group", [0, 32])
def test_small_and_large_norms(size, group):
    """Whose scales lie near the least one, and norms near fp32's largest."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(3)
    tokens, dim = 3000, 776
    x = torch.randn(tokens, dim, generator=gen, device="cuda").bfloat16()
    # many values on ties, and far below the row's largest
    x = x * torch.exp2(-torch.randint(0, 16, (tokens, dim), generator=gen, device="cuda"))
    w = (1.0 + 0.2 * torch.randn(dim, generator=gen, device="cuda")).bfloat16().float() * size
    y = ops.rms_norm(x, w, out_dtype=torch.float32).cpu()
    q, scales = ops.rms_norm_fp8(x, w, group=group)
    want, want_scales = _want(torch, y, group)
    assert torch.equal(scales.cpu(), want_scales)
    assert torch.equal(q.cpu().view(torch.uint8), want.view(torch.uint8))
