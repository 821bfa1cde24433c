"""Operands that are column slices of one buffer: their rows lie between each other and
share no element."""

import math

import pytest

import ops_reference as R
from gpu_harness import torch_cuda
from test_gpu_ortho import SPLIT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", [64, 37])
def test_matrices_of_a_fused_weight(dtype, cols):
    """Three matrices side by side, each made orthogonal by itself: into slices of another
    buffer, of the same one, and in place."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    dtype = getattr(torch, dtype)
    tol = SPLIT if dtype == torch.float32 else 3e-3
    gen = torch.Generator(device="cuda").manual_seed(1)
    fused = torch.randn(96, 6 * cols, generator=gen, device="cuda").to(dtype)
    fused[:, 3 * cols:] = 7.0
    part = lambda t, i: t[:, i * cols:(i + 1) * cols]  # noqa: E731
    want = [R.newton_schulz(part(fused, i)) for i in range(3)]
    out = torch.full_like(fused, math.nan)
    ops.Orthogonalizer([part(fused, i) for i in range(3)], [part(out, i) for i in range(3)]).run()
    assert out[:, 3 * cols:].isnan().all() and bool((fused[:, 3 * cols:] == 7).all())
    for i in range(3):
        assert R.relative(part(out, i), want[i]) < tol
    before = fused[:, :3 * cols].clone()
    ops.Orthogonalizer([part(fused, i) for i in range(3)],
                       [part(fused, 5 - i) for i in range(3)]).run()
    assert torch.equal(fused[:, :3 * cols], before)
    for i in range(3):
        assert torch.equal(part(fused, 5 - i), part(out, i))
    ops.Orthogonalizer([part(fused, i) for i in range(3)], [part(fused, i) for i in range(3)]).run()
    for i in range(3):
        assert torch.equal(part(fused, i), part(out, i))


def test_lookup_and_its_gradient_beside_their_operands():
    torch = torch_cuda()
    from paper_1904_00962_amd import _lib, ops
    gen = torch.Generator(device="cuda").manual_seed(2)
    ids = torch.randint(0, 50, (50,), generator=gen, device="cuda")
    both = torch.randn(50, 80, generator=gen, device="cuda")
    table = both[:, :40].clone()
    ops.embedding(ids, both[:, :40], out=both[:, 40:])
    assert torch.equal(both[:, :40], table) and torch.equal(both[:, 40:], table[ids])
    rows = both[:, 40:].clone()
    ops.embedding_grad(ids, both[:, 40:], both[:, :40])
    alone = torch.empty_like(table)
    ops.embedding_grad(ids, rows, alone)
    assert torch.equal(both[:, :40], alone) and torch.equal(both[:, 40:], rows)
    with pytest.raises(_lib.LambError):
        ops.embedding(ids, both[:, :41], out=both[:, 39:])


def test_gradients_of_the_loss_in_slices():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(3)
    both = torch.randn(70, 96, generator=gen, device="cuda").bfloat16()
    h, gh = both[:, :48], both[:, 48:]
    tables = torch.randn(90, 96, generator=gen, device="cuda").bfloat16()
    w, gw = tables[:, 48:], tables[:, :48]
    t = torch.randint(0, 90, (70,), generator=gen, device="cuda")
    _, _, lse = ops.linear_cross_entropy(h, w, t)
    a, b = torch.empty(70, 48, dtype=both.dtype, device="cuda"), torch.empty_like(gw)
    ops.linear_cross_entropy_grad(h, w, t, lse, a, b)
    ops.linear_cross_entropy_grad(h, w, t, lse, gh, gw)
    assert torch.equal(gh, a) and torch.equal(gw, b)
