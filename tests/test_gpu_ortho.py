"""Newton-Schulz orthogonalization and the Muon step on the GPU against their
formulas in 64 bits.

Tolerances. A step rounds X, A and P once each, by u in the root mean square
(relative): 2^-13 for one 16-bit float of 11 significant bits, 2^-24 for a pair of
them. A relative error e of a singular value s becomes |s f'(s) / f(s)| e under
f(s) = a s + b s^3 + c s^5, 1.5 on average over the singular values that the default
coefficients lead to (0.7 to 1.2; 5 at the end near 1.2). Five steps then leave about
sqrt(3) u (1 + 1.5 + ... + 1.5^4) = 23 u: 2.8e-3 and 1.4e-6. Rounding the result to
bfloat16 adds 1.7e-3. The tests allow about three times these. Singular values that
span decades cost more: the small ones keep the absolute error of the large ones.
"""

import math

import pytest

import ops_reference as R
from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu

HALF, SPLIT = 9e-3, 5e-6
SHAPES = [(1, 1), (1, 7), (7, 1), (1, 1000), (5000, 1), (2, 2), (9, 8), (16, 16), (63, 65),
          (64, 64), (65, 63), (128, 256), (129, 127), (147, 64), (257, 511), (512, 100),
          (300, 1100), (1000, 513)]


def _make(torch, shapes, dtype, seed=0, sigma=1e-3):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(r, c, generator=gen, device="cuda").mul_(sigma).to(dtype)
            for r, c in shapes]


@pytest.mark.parametrize("src,dst,precision", [
    ("float32", "float32", None), ("bfloat16", "bfloat16", None), ("float32", "bfloat16", None),
    ("bfloat16", "float32", None), ("float32", "float32", "half"),
    ("float32", "bfloat16", "split")])
def test_every_shape_in_one_list(src, dst, precision):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gs = _make(torch, SHAPES, getattr(torch, src))
    outs = [torch.full(g.shape, math.nan, dtype=getattr(torch, dst), device="cuda") for g in gs]
    ops.Orthogonalizer(gs, outs, precision=precision).run()
    split = precision == "split" or (precision is None and dst == "float32")
    tol = SPLIT if split else HALF
    if split and dst == "bfloat16":
        tol = 3e-3
    for g, o in zip(gs, outs):
        assert R.relative(o, R.newton_schulz(g)) < tol, tuple(g.shape)


@pytest.mark.parametrize("dtype,tol", [("float32", SPLIT), ("bfloat16", HALF)])
def test_lists_that_take_the_larger_tiles(dtype, tol):
    """Lists long enough to fill the device take other tile shapes; all of the matrices
    differ, so a tile that went to another matrix shows."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    for shapes in ([(260, 520)] * 60 + [(520, 130)] * 20, [(1030, 1030)] * 14 + [(776, 1290)] * 6):
        gs = _make(torch, shapes, getattr(torch, dtype), seed=3)
        outs = ops.Orthogonalizer(gs).run()
        for i in list(range(0, len(gs), 7)) + [len(gs) - 1]:
            assert R.relative(outs[i], R.newton_schulz(gs[i])) < tol, (i, shapes[i])


@pytest.mark.parametrize("dtype,count,tol", [("float32", 80, SPLIT), ("bfloat16", 320, HALF)])
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5, 6, 7])
def test_long_lists_of_long_matrices_iterate_in_chains(dtype, count, tol, steps):
    """Enough work in matrices twice as long as wide that their iterations run on the
    short side; square ones in the same list do not. Some are of low rank and noise, a
    few with singular values over four decades (held to the tolerance of those)."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    shapes = [(256, 1024)] * count + [(1030, 257), (515, 256), (300, 300), (259, 130)]
    gs = _make(torch, shapes, getattr(torch, dtype), seed=steps)
    gen = torch.Generator(device="cuda").manual_seed(7)
    u, v = (torch.randn(256, 16, generator=gen, device="cuda"),
            torch.randn(16, 1024, generator=gen, device="cuda"))
    gs[3].add_((u @ v).to(gs[3].dtype), alpha=2e-4)
    gs[5].mul_(torch.logspace(0, -4, 256, device="cuda")[:, None].to(gs[5].dtype))
    outs = ops.Orthogonalizer(gs, steps=steps).run()
    for i in (0, 1, 3, 5, count - 1, count, count + 1, count + 2, count + 3):
        loose = 5 if i in (3, 5) else 1
        err = R.relative(outs[i], R.newton_schulz(gs[i], steps))
        assert err < loose * tol * (1 if steps <= 5 else 2), (i, shapes[i], err)


@pytest.mark.parametrize("steps", [1, 2, 8])
def test_steps_and_coefficients(steps):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gs = _make(torch, [(96, 200), (200, 96)], torch.float32)
    for coef in (R.COEF, (1.5, -0.5, 0.0), (1.875, -1.25, 0.375)):
        outs = ops.Orthogonalizer(gs, steps=steps, coefficients=coef).run()
        for g, o in zip(gs, outs):
            want = R.newton_schulz(g, steps, coef)
            assert R.relative(o, want) < SPLIT * (1 if steps <= 5 else 4), (coef, tuple(g.shape))


def test_strides_views_and_in_place():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(5)
    wide = torch.randn(100, 333, generator=gen, device="cuda")
    store = torch.full((100, 700), 7.0, device="cuda")
    # an odd offset, rows 333 and 700 elements apart
    g, o = wide[3:90, 5:150], store[3:90, 9:154]
    want = R.newton_schulz(g)
    ops.Orthogonalizer([g], [o]).run()
    assert R.relative(o, want) < SPLIT
    untouched = store.clone()
    untouched[3:90, 9:154] = 7.0
    assert torch.equal(untouched, torch.full_like(untouched, 7.0))
    # aligned, and in place
    for dtype, tol in ((torch.float32, SPLIT), (torch.bfloat16, HALF)):
        a = torch.randn(64, 128, generator=gen, device="cuda").to(dtype)
        want = R.newton_schulz(a)
        ops.Orthogonalizer([a], [a]).run()
        assert R.relative(a, want) < tol


def test_zero_nan_and_scale():
    """A zero matrix stays 0; a matrix that holds a NaN or an infinity becomes NaN and
    touches no other; the result does not depend on the input's scale."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gs = _make(torch, [(40, 60)] * 6, torch.float32, seed=9)
    gs[0].zero_()
    gs[1][3, 4] = math.nan
    gs[2][39, 59] = math.inf
    gs[4].copy_(gs[3]).mul_(2.0 ** 60)
    gs[5].copy_(gs[3]).mul_(1e18)
    outs = ops.Orthogonalizer(gs).run()
    assert not outs[0].any()
    assert outs[1].isnan().all() and outs[2].isnan().all()
    want = R.newton_schulz(gs[3])
    for o in outs[3:]:
        assert R.relative(o, want) < SPLIT
    tiny = [gs[3] * 1e-30]
    o = ops.Orthogonalizer(tiny, eps=0.0).run()[0]
    assert R.relative(o, R.newton_schulz(tiny[0], eps=0.0)) < SPLIT


@pytest.mark.parametrize("decades", [2, 5])
def test_singular_values_that_span_decades(decades):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator().manual_seed(decades)
    u, _, v = torch.linalg.svd(torch.randn(160, 240, generator=gen, dtype=torch.float64),
                               full_matrices=False)
    s = 10.0 ** torch.linspace(0.0, -float(decades), 160, dtype=torch.float64)
    g = (u * s @ v).float().cuda()
    want = R.newton_schulz(g)
    # a relative error of u of the largest is u / s of the others, on those that grow
    # to the result's size: 3.4445^5 = 485 times at most
    assert R.relative(ops.Orthogonalizer([g]).run()[0], want) < 4e-5
    assert R.relative(ops.Orthogonalizer([g], precision="half").run()[0], want) < 5e-2


def test_same_bits_twice_on_another_stream_and_in_a_graph():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gs = _make(torch, [(130, 70), (70, 300), (256, 256)], torch.bfloat16)
    plan = ops.Orthogonalizer(gs)
    first = [o.clone() for o in plan.run()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plan.run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, plan.outputs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run()
    for k in range(3):
        fresh = _make(torch, [tuple(g.shape) for g in gs], torch.bfloat16, seed=20 + k)
        for g, f in zip(gs, fresh):
            g.copy_(f)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [o.clone() for o in plan.outputs]
        plan.run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, plan.outputs)), k


def _muon_state(torch, shapes, g_dtype, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    xs = [torch.randn(*s, generator=gen, device="cuda").mul_(0.02) for s in shapes]
    gs = [torch.randn(*s, generator=gen, device="cuda").mul_(1e-3).to(g_dtype) for s in shapes]
    ms = [torch.randn(*s, generator=gen, device="cuda").mul_(2e-4) for s in shapes]
    return xs, gs, ms


MUON_SHAPES = [(64, 147), (200, 96), (33, 1), (1, 40), (256, 64, 3, 3), (8, 8)]


@pytest.mark.parametrize("g_dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("nesterov,scale,precision,masked", [
    (True, "rms", "split", False), (False, "spectral", "split", True), (True, "unit", "half", False)])
def test_muon_steps(g_dtype, nesterov, scale, precision, masked):
    """x moves by lr s O: its error is that of O in that share, and the rounding of x."""
    torch = torch_cuda()
    from paper_1904_00962_amd import Muon
    xs, gs, ms = _muon_state(torch, MUON_SHAPES, getattr(torch, g_dtype))
    mask = [i % 2 == 0 for i in range(len(xs))] if masked else None
    opt = Muon(xs, gs, lr=0.02, momentum=0.9, weight_decay=0.3, nesterov=nesterov, scale=scale,
               precision=precision, m=ms, wd_mask=mask, grad_scale=0.25)
    for k in range(2):
        want = [R.muon_step(x.reshape(x.shape[0], -1), g.reshape(x.shape[0], -1),
                            m.reshape(x.shape[0], -1), 0.02 * (k + 1), 0.9, 0.3, nesterov, scale,
                            grad_scale=0.25, wd=mask is None or mask[i])
                for i, (x, g, m) in enumerate(zip(xs, gs, ms))]
        before = [x.clone() for x in xs]
        opt.step(lr=0.02 * (k + 1))
        for x, m, old, (wx, wm) in zip(xs, ms, before, want):
            assert R.relative(m.reshape(wm.shape), wm) < 3e-7
            moved = wx - old.reshape(wx.shape).double()
            got = x.reshape(wx.shape).double() - old.reshape(wx.shape).double()
            rounding = 2.0 ** -24 * float(torch.linalg.vector_norm(wx))
            off = float(torch.linalg.vector_norm(got - moved))
            tol = SPLIT if precision == "split" else HALF
            assert off < tol * float(torch.linalg.vector_norm(moved)) + 3 * rounding
        gs[0].copy_(gs[0].flip(0))
    assert opt.t == 2
    state = opt.state_dict()
    opt.load_state_dict(state)
    assert state["step"] == 2 and torch.equal(state["m"][2], opt.m[2])


def test_muon_skips_a_step_with_a_nonfinite_gradient():
    torch = torch_cuda()
    from paper_1904_00962_amd import Muon
    xs, gs, ms = _muon_state(torch, [(40, 24), (24, 72)], torch.bfloat16)
    opt = Muon(xs, gs, m=ms, skip_nonfinite=True, lr=0.01)
    good = gs[1].clone()
    for bad in (math.nan, math.inf, None, -math.inf, None):
        gs[1].copy_(good)
        if bad is not None:
            gs[1][23, 71] = bad
        before = [t.clone() for t in xs + ms]
        opt.step()
        torch.cuda.synchronize()
        same = [torch.equal(a, b) for a, b in zip(before, xs + ms)]
        assert int(opt.found_nonfinite) == (bad is not None)
        assert all(same) if bad is not None else not any(same)


def test_muon_without_the_check_spreads_only_within_a_matrix():
    torch = torch_cuda()
    from paper_1904_00962_amd import Muon
    xs, gs, ms = _muon_state(torch, [(40, 24), (24, 72)], torch.float32)
    gs[0][1, 1] = math.nan
    want, _ = R.muon_step(xs[1], gs[1], ms[1], 0.01, 0.95)
    Muon(xs, gs, m=ms, lr=0.01).step()
    assert xs[0].isnan().all()
    assert R.relative(xs[1], want) < 1e-6


def test_muon_schedule():
    torch = torch_cuda()
    from paper_1904_00962_amd import Muon, _lib
    xs, gs, ms = _muon_state(torch, [(16, 16)], torch.float32)
    stages = [(10, 4, 0.1, 1.0)]
    opt = Muon(xs, gs, m=ms, schedule=stages)
    want, _ = R.muon_step(xs[0], gs[0], ms[0], _lib.lamb_lr_at(stages, 1), 0.95)
    opt.step()
    assert R.relative(xs[0], want) < 1e-6


@pytest.mark.parametrize("fields,words", [
    (dict(steps=0), "steps"), (dict(steps=65), "steps"), (dict(eps=-1.0), "eps"),
    (dict(a=math.nan), "finite"), (dict(reserved=1), "reserved"),
    (dict(a=1e4), "polynomial"), (dict(a=3.4445, b=0.0, c=0.0), "singular value"),
])
def test_iteration_bounds(fields, words):
    """Among them coefficients that let the iteration leave the range of its operands."""
    torch = torch_cuda()
    from paper_1904_00962_amd import _lib, _ops, ops
    g = torch.ones(4, 8, device="cuda")
    o = ops.Orthogonalizer([g])
    with pytest.raises(_lib.LambError, match=words):
        _ops.lamb_orthogonalize(o.plan, _ops.lamb_ns_params_init(**fields), 0)


def test_muon_scalars():
    torch = torch_cuda()
    from paper_1904_00962_amd import _lib, _ops
    x, m = torch.ones(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    g = torch.ones(4, 8, device="cuda")
    row = (x.data_ptr(), g.data_ptr(), m.data_ptr(), 4, 8, 1)
    plan = _ops.lamb_muon_plan_create([row], _ops.LAMB_DTYPE_F32, _ops.LAMB_NS_HALF)
    for fields in (dict(lr=-1.0), dict(lr=math.nan), dict(momentum=1.0), dict(weight_decay=-0.1),
                   dict(grad_scale=0.0), dict(nesterov=2), dict(scale=3), dict(skip_nonfinite=-1),
                   dict(reserved=1)):
        with pytest.raises(_lib.LambError):
            _ops.lamb_muon_step(plan, _ops.lamb_muon_hparams_init(**fields), 0)
    torch.cuda.synchronize()
    plan.close()
    assert x.eq(1).all() and m.eq(0).all()


def test_small_matrices_are_no_further_off_than_fp32():
    """Their few roundings do not average out, so the split products keep every part."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    a, b, c = ops.COEFFICIENTS
    for shape in ((12, 10), (45, 45), (59, 161)):
        gs = _make(torch, [shape] * 100, torch.float32, seed=5)
        ours, plain = [], []
        for g, got in zip(gs, ops.Orthogonalizer(gs, precision="split").run()):
            x = g.mT if g.shape[0] > g.shape[1] else g
            x = x / (torch.linalg.vector_norm(x) + 1e-7)
            for _ in range(5):
                gram = x @ x.mT
                x = a * x + (b * gram + c * (gram @ gram)) @ x
            want = R.newton_schulz(g)
            ours.append(R.relative(got, want))
            plain.append(R.relative(x.mT if g.shape[0] > g.shape[1] else x, want))
        assert sorted(ours)[50] <= sorted(plain)[50]
