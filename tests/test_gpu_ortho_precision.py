"""What the precisions of the Newton-Schulz products promise on matrices whose singular
values are far apart, as a network's gradients and momenta have them.

Tolerances. X has norm 1 at first (Frobenius, here throughout). Rounding it by u of each
entry at most is an error of u, and every later step multiplies what lies beside the
large singular values by up to a = 3.4445. Step k's rounding of an X of norm at most 1.2
thus ends as 1.2 u a^(5 - k + 1); independent of one another, the five add up in squares:
1.2 u 506 = 607 u. A's and P's roundings hit what X is large in, not what is small. u is
2^-11 for one 16-bit float and 2^-22 for two: errors of 0.30 and 1.5e-4, to which the
fp32 sums of the split products add as much again at most. A bf16 result is rounded by
its type beside that; an error e before it moves that by e again at most."""

import math

import pytest

import ops_reference as R
from gpu_harness import torch_cuda
from test_gpu_ortho import HALF, _make

pytestmark = pytest.mark.gpu

A = R.COEF[0]
GROWTH = 1.2 * math.sqrt(sum(A ** (2 * k) for k in range(1, 6)))
HALF_OFF, SPLIT_OFF = GROWTH * 2.0 ** -11, 2 * GROWTH * 2.0 ** -22


def _spectrum(torch, kind, rows, cols, seed=1):
    gen = torch.Generator().manual_seed(seed)
    normal = lambda r, c: torch.randn(r, c, generator=gen, dtype=torch.float64)  # noqa: E731
    if kind.startswith("decades"):
        u, _, v = torch.linalg.svd(normal(rows, cols), full_matrices=False)
        s = 10.0 ** torch.linspace(0.0, -float(kind[7:]), min(rows, cols), dtype=torch.float64)
        return (u * s @ v).float().cuda()
    rank, noise = {"one": (1, 1e-3), "few": (16, 2e-3), "some": (32, 1e-2)}[kind]
    low = normal(rows, rank) @ normal(rank, cols) / math.sqrt(rank)
    return (low + noise * normal(rows, cols)).float().cuda()


KINDS = ["decades3", "decades6", "one", "few", "some"]


def _off(torch, got, want):
    return float(torch.linalg.vector_norm(got.double() - want))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [(128, 512), (256, 256), (240, 160)])
def test_results_keep_their_type_s_accuracy_unless_half_is_asked_for(kind, rows, cols):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    g = _spectrum(torch, kind, rows, cols)
    for src, dst in ((torch.float32, torch.float32), (torch.float32, torch.bfloat16),
                     (torch.bfloat16, torch.bfloat16)):
        x = g.to(src)
        want = R.newton_schulz(x)
        out = torch.empty(g.shape, dtype=dst, device="cuda")
        ops.Orthogonalizer([x], [out]).run()
        alone = 0.0 if dst == torch.float32 else _off(torch, want.to(dst), want)
        assert _off(torch, out, want) <= alone + 2 * SPLIT_OFF, (src, dst)


def test_the_precision_does_not_go_by_the_list():
    """One narrow matrix or a short one changes nothing for the others."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    wide = _make(torch, [(256, 256)] * 3, torch.bfloat16)
    for more in ([], _make(torch, [(32, 512)], torch.bfloat16), _make(torch, [(1, 9)],
                                                                      torch.bfloat16)):
        assert ops.Orthogonalizer(wide + more).precision == "split"
    assert ops.Orthogonalizer(wide, precision="half").precision == "half"


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("count", [1, 320])  # 320: in chains
def test_half_is_off_by_its_rounding_grown(kind, count):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    g = _spectrum(torch, kind, 256, 1024)
    want = R.newton_schulz(g)
    outs = ops.Orthogonalizer([g] * count, [torch.empty_like(g) for _ in range(count)],
                              precision="half").run()
    assert _off(torch, outs[0], want) <= HALF_OFF
    assert all(torch.equal(o, outs[0]) for o in outs)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5])
def test_half_lists_of_every_tile(steps):
    """Lists that take each tile shape and, the last, chains; all of the matrices differ."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    for shapes in ([(64, 64), (129, 127), (512, 100)], [(260, 520)] * 60 + [(520, 130)] * 20,
                   [(1030, 1030)] * 14 + [(776, 1290)] * 6,
                   [(256, 1024)] * 320 + [(1030, 257), (300, 300)]):
        gs = _make(torch, shapes, torch.bfloat16, seed=steps)
        outs = ops.Orthogonalizer(gs, steps=steps, precision="half").run()
        for i in list(range(0, len(gs), 37)) + [len(gs) - 1]:
            assert R.relative(outs[i], R.newton_schulz(gs[i], steps)) < HALF, (i, shapes[i])


@pytest.mark.parametrize("momentum", [0.9, 0.95, 0.99, 0.999])
@pytest.mark.parametrize("nesterov", [False, True])
def test_muons_momentum_is_the_one_asked_for(momentum, nesterov):
    """m, rounded once (2^-24 of it): within 2^-23 of the sum of its terms' magnitudes."""
    torch = torch_cuda()
    from paper_1904_00962_amd import Muon
    gen = torch.Generator(device="cuda").manual_seed(3)
    for scale in (0.0, 1e-3, 1.0):  # of the old momentum; 0: m is (1 - momentum) g
        x, g, m = (torch.randn(70, 90, generator=gen, device="cuda") for _ in range(3))
        m.mul_(scale)
        want = momentum * m.double() + (1.0 - momentum) * g.double()
        size = momentum * m.double().abs() + (1.0 - momentum) * g.double().abs()
        Muon([x], [g], m=[m], momentum=momentum, nesterov=nesterov).step()
        assert bool(((m.double() - want).abs() <= 2.0 ** -23 * size).all())


@pytest.mark.parametrize("sigma", [1e-30, 1e-34, 1e-37, 1e-40, 1e-43])
@pytest.mark.parametrize("shape", [(40, 60), (1, 7), (3, 2)])
def test_without_eps_no_matrix_is_too_small(sigma, shape):
    """Down to denormal entries, which the input's rounding makes other numbers; the result
    is that of these numbers, at any scale."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(2)
    g = (torch.randn(shape, generator=gen, dtype=torch.float64, device="cuda") * sigma).float()
    assert bool(g.any())
    o = ops.Orthogonalizer([g], eps=0.0).run()[0]
    assert _off(torch, o, R.newton_schulz(g, eps=0.0)) <= SPLIT_OFF
