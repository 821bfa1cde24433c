"""Norms of lists of gradients and clipping by them. Norms are sums in fp64 of at most a few
thousand roundings in a row: 2^-53 each of a sum of like signs, 1e-12 with room. A clipped
gradient is compared with exactly its product, in fp32, with the factor that the norm
gives, rounded to its type."""

import math

import pytest

from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu

SIZES = [[1], [7], [8], [9], [2047], [2048], [2049], [65537, 1, 0, 3, 300001, 8, 0, 4095],
         [1 << 20] * 3 + [5] * 70, [0], [0, 0, 12], [1] * 1500]


def _grads(torch, sizes, gen, kind="mixed", gap=0, sigma=1.0):
    """Tensors that lie one after another in a buffer of each type, ``gap`` elements between
    them, and the buffers."""
    types = {"mixed": (torch.float32, torch.bfloat16), "f32": (torch.float32,),
             "bf16": (torch.bfloat16,)}[kind]
    room = sum(sizes) + gap * len(sizes) + 1
    flat = {t: torch.randn(room, generator=gen, device="cuda").mul_(sigma).to(t) for t in types}
    at, got = dict.fromkeys(types, 1), []
    for i, n in enumerate(sizes):
        t = types[i % len(types)]
        got.append(flat[t][at[t]:at[t] + n])
        at[t] += n + gap
    return got, flat


def _norms(torch, grads, kind):
    per = [g.double().abs() for g in grads]
    if kind == "l2":
        return torch.stack([p.square().sum().sqrt() for p in per])
    if kind == "l1":
        return torch.stack([p.sum() for p in per])
    return torch.stack([p.max() if p.numel() else p.sum() for p in per])


def _total(norms, kind):
    return {"l2": norms.square().sum().sqrt(), "l1": norms.sum(), "linf": norms.max()}[kind]


def _near(a, b, kind):
    return bool((a == b).all() if kind == "linf" else ((a - b).abs() <= 1e-12 * b).all())


def _factor(torch, total, max_norm, scale=1.0):
    over = math.isfinite(total) and abs(scale) * total > max_norm
    f = math.copysign(max_norm / total, scale) if over else scale
    return torch.tensor(f, dtype=torch.float64).float().cuda()


@pytest.mark.parametrize("sizes", SIZES, ids=[str(k) for k in range(len(SIZES))])
@pytest.mark.parametrize("kind", ["l2", "l1", "linf"])
def test_norms(sizes, kind):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(len(sizes))
    for types in ("mixed", "f32", "bf16"):
        grads, _ = _grads(torch, sizes, gen, types)
        plan = ops.GradNorm(grads, norm=kind)
        total = plan.run()
        want = _norms(torch, grads, kind)
        assert _near(plan.norms, want, kind) and _near(total, _total(want, kind), kind)
        assert total is plan.total and total.dtype == torch.float64
        bits = plan.norms.clone(), total.clone()
        plan.run()
        assert torch.equal(plan.norms, bits[0]) and torch.equal(plan.total, bits[1])


def test_squares_past_the_range_of_fp32():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(1)
    for sigma in (1e30, 1e-30, 1e-42):
        grads, _ = _grads(torch, [5000, 3], gen, "f32", sigma=sigma)
        plan = ops.GradNorm(grads)
        assert _near(plan.run(), _total(_norms(torch, grads, "l2"), "l2"), "l2")


@pytest.mark.parametrize("sizes", SIZES, ids=[str(k) for k in range(len(SIZES))])
def test_clip(sizes):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(len(sizes))
    for types in ("mixed", "bf16"):
        for out_type in (None, torch.float32, torch.bfloat16):
            for limit, scale in ((1.0, 1.0), (1.0, -0.25), (1e9, 1.0), (1e9, 0.5), (0.0, 1.0),
                                 (math.inf, 1.0)):
                grads, flat = _grads(torch, sizes, gen, types, gap=3)
                old = {t: f.clone() for t, f in flat.items()}
                before = [g.clone() for g in grads]
                outputs = None if out_type is None else [
                    torch.full((g.numel(),), math.nan, dtype=out_type, device="cuda")
                    for g in grads]
                plan = ops.GradNorm(grads, outputs)
                total = float(plan.clip(limit, scale=scale))
                assert total == float(ops.GradNorm(before).run())
                f = _factor(torch, total, limit, scale)
                for g, o in zip(before, plan.outputs):
                    assert torch.equal(o, (g.float() * f).to(o.dtype))
                assert int(plan.found_nonfinite) == 0
                # what lies between the tensors is as it was
                for t in flat:
                    kept = torch.ones(len(flat[t]), dtype=torch.bool, device="cuda")
                    for g in grads:
                        if g.dtype == t and out_type is None:
                            kept[g.storage_offset():g.storage_offset() + g.numel()] = False
                    assert torch.equal(flat[t][kept], old[t][kept])


def test_clipped_gradients_keep_the_limit():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(2)
    for kind in ("l2", "l1", "linf"):
        grads, _ = _grads(torch, [70000, 300, 5], gen, "f32")
        plan = ops.GradNorm(grads, norm=kind)
        before = float(plan.clip(0.5))
        assert before > 0.5
        # the factor's rounding to fp32 and the products'
        assert abs(float(plan.run()) - 0.5) <= 0.5 * 2.0 ** -22


def test_a_scale_whose_norm_passes_every_type():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(8)
    grads, _ = _grads(torch, [3000], gen, "f32", sigma=1e10)
    before = grads[0].double()
    plan = ops.GradNorm(grads)
    total = float(plan.clip(2.0, scale=-1e305))
    assert float(torch.linalg.vector_norm(grads[0].double() + before * (2.0 / total))) <= 2.0 ** -22


def test_results_of_a_plan_made_on_a_busy_stream():
    """A call on another stream than the one that made the plan's results."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    g = torch.ones(5000, device="cuda")
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(a):
        torch.cuda._sleep(5_000_000)
        plan = ops.GradNorm([g], norm="l1")
    with torch.cuda.stream(b):
        plan.run()
    torch.cuda.synchronize()
    assert float(plan.total) == 5000.0 and float(plan.norms[0]) == 5000.0


def test_totals_that_are_no_number():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(3)
    for kind in ("l2", "l1", "linf"):
        for bad in (math.nan, math.inf, -math.inf):
            grads, _ = _grads(torch, [3000, 40, 0, 9], gen)
            grads[1][17] = bad
            before = [g.clone() for g in grads]
            plan = ops.GradNorm(grads, norm=kind)
            total = float(plan.clip(0.1))
            same = (lambda v: math.isnan(v)) if math.isnan(bad) else (lambda v: v == math.inf)
            assert same(total) and same(float(plan.norms[1])) and int(plan.found_nonfinite) == 1
            assert bool(plan.norms[[0, 2, 3]].isfinite().all())
            for a, b in zip(before, grads):
                assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))
            grads[1][17] = 1.0
            plan.clip(0.1)
            assert int(plan.found_nonfinite) == 0
    grads[0][5], grads[1][2] = math.inf, math.nan
    assert math.isnan(float(plan.run()))


def test_a_norm_over_workers():
    """Two halves of one list, their common norm from the sum of squares of both."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(4)
    grads, _ = _grads(torch, [5000, 77, 1234, 8], gen, "f32")
    both = ops.GradNorm([g.clone() for g in grads])
    parts = [ops.GradNorm(grads[:2]), ops.GradNorm(grads[2:])]
    total = torch.stack([p.run().square() for p in parts]).sum().sqrt()
    both.clip(1.0)
    for p in parts:
        assert p.clip(1.0, total=total) is total
    for a, b in zip(grads, both.outputs):
        assert bool(((a - b).abs() <= 2.0 ** -22 * b.abs()).all())


def test_streams_and_graphs():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(5)
    grads, _ = _grads(torch, [300000, 17, 4001], gen)
    outputs = [torch.empty(g.numel(), dtype=torch.bfloat16, device="cuda") for g in grads]
    plan = ops.GradNorm(grads, outputs)
    plan.clip(1.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.clip(1.0)
    side = torch.cuda.Stream()
    for k in range(4):
        for g in grads:
            g.copy_(torch.randn(g.numel(), generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        held = [t.clone() for t in (*outputs, plan.norms, plan.total)]
        for o in outputs:
            o.zero_()
        plan.total.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(1_000_000)
            plan.run()
        plan.clip(1.0)  # waits for the call on the other stream
        torch.cuda.synchronize()
        for a, b in zip(held, (*outputs, plan.norms, plan.total)):
            assert torch.equal(a, b), k


def test_more_elements_than_32_bits():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    n = (1 << 32) + 11
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[1 << 31], g[n - 1] = 3.0, 4.0, 12.0
    plan = ops.GradNorm([g])
    assert float(plan.clip(6.5)) == 13.0
    assert [float(g[i]) for i in (0, 1 << 31, n - 1)] == [1.5, 2.0, 6.0]


@pytest.mark.parametrize("optimizer", ["LAMB", "LARS", "Muon"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_the_optimizers_limit(optimizer, dtype):
    """A step with max_grad_norm is one after the gradients were clipped by hand."""
    torch = torch_cuda()
    from paper_1904_00962_amd import LAMB, LARS, Muon, ops
    kind = {"LAMB": LAMB, "LARS": LARS, "Muon": Muon}[optimizer]
    gen = torch.Generator(device="cuda").manual_seed(6)
    shapes = [(64, 48), (7, 9), (33, 128)] + ([] if optimizer == "Muon" else [(31,)])
    sides = []
    for limit in (0.75, None):
        gen.manual_seed(6)
        xs = [torch.randn(*s, generator=gen, device="cuda") for s in shapes]
        gs = [torch.empty(*s, dtype=getattr(torch, dtype), device="cuda") for s in shapes]
        sides.append((xs, gs, kind(xs, gs, lr=0.01, grad_scale=0.5, skip_nonfinite=True,
                                   max_grad_norm=limit)))
    (xs, gs, opt), (ys, hs, plain) = sides
    by_hand = ops.GradNorm(hs)
    for step, sigma in enumerate((1.0, 1e-4, 3.0, 1.0)):
        new = [torch.randn(*s, generator=gen, device="cuda") * sigma for s in shapes]
        if step == 2:
            new[1][0, 0] = math.nan
        for g, h, v in zip(gs, hs, new):
            g.copy_(v), h.copy_(v)
        opt.step()
        total = by_hand.clip(1.5)  # of gradients that the step halves
        plain.step()
        torch.cuda.synchronize()
        assert torch.equal(opt.grad_norm.nan_to_num(-1.0), total.nan_to_num(-1.0))
        assert int(opt.found_nonfinite) == (step == 2)
        for a, b in zip(xs + gs, ys + hs):
            assert torch.equal(a.nan_to_num(5.0), b.nan_to_num(5.0))
    assert plain.grad_norm is None
    opt.close(), plain.close()


def test_refusals():
    torch = torch_cuda()
    from paper_1904_00962_amd import LAMB, _lib, ops
    g = torch.zeros(64, device="cuda")
    for call in (lambda: ops.GradNorm([g.half()]), lambda: ops.GradNorm([g], [g.double()])):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ops.GradNorm([]), lambda: ops.GradNorm([g.cpu()]),
                 lambda: ops.GradNorm([g[::2]]), lambda: ops.GradNorm([g], [g[:3]]),
                 lambda: ops.GradNorm([g], []), lambda: ops.GradNorm([g], norm="l3"),
                 lambda: LAMB([g.clone()], [g], max_grad_norm=0.0),
                 lambda: LAMB([g.clone()], [g], max_grad_norm=math.nan)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ops.GradNorm([g, g]), lambda: ops.GradNorm([g[:40], g[32:]]),
                 lambda: ops.GradNorm([g[:32]], [g[16:48]])):
        with pytest.raises(_lib.LambError) as e:
            call()
        assert e.value.status == _lib.LAMB_EOVERLAP
    plan = ops.GradNorm([g])
    for call in (lambda: plan.clip(-1.0), lambda: plan.clip(math.nan),
                 lambda: plan.clip(1.0, scale=math.inf)):
        with pytest.raises(_lib.LambError) as e:
            call()
        assert e.value.status == _lib.LAMB_EINVAL
    with pytest.raises(TypeError):
        plan.clip(1.0, total=torch.zeros((), device="cuda"))
    with pytest.raises(ValueError):
        plan.clip(1.0, total=torch.zeros((), dtype=torch.float64))
    plan.close()
    with pytest.raises(_lib.LambError):
        plan.run()
