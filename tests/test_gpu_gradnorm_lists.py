"""Norms and clipping of lists as long as models have them: more chunks than one launch
joins, chunks of every length, several tensors that begin anywhere and take many chunks,
and lists past the size up to which the norms' loads stay in the caches. Norms are sums in
fp64 of at most a few hundred roundings in a row, 2^-53 each: 1e-12 with room. A clipped
gradient is the fp32 product with the factor that the norm gives, rounded to its type."""

import math

import pytest

from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu

# elements of all tensors: chunks of 8192, 10240, 14336 and 16384, all past 640 of them
TOTALS = [6_000_000, 20_000_000, 29_000_000, 40_000_000]
PAST_THE_CACHES = 210_000_000  # 840 MB of fp32


def _sizes(total):
    small = [1, 16384, 0, 16385, 8193, 5, 3 * 8192 + 1, 2049, 14335, 10241, 7]
    part = [total * k // 100 | 1 for k in (31, 7, 2, 23)]
    return [part[0], *small[:4], part[1], *small[4:8], part[2], part[3], *small[8:],
            total - sum(part) - sum(small)]


def _grads(torch, total, kind, gen):
    types = {"mixed": (torch.float32, torch.bfloat16), "f32": (torch.float32,),
             "bf16": (torch.bfloat16,)}[kind]
    sizes = _sizes(total)
    assert min(sizes) >= 0 and sum(sizes) == total
    which = [types[i % len(types)] for i in range(len(sizes))]
    flat = {t: torch.randn(sum(n + 3 for n, u in zip(sizes, which) if u == t) + 1, generator=gen,
                           device="cuda").to(t) for t in types}
    at, grads = dict.fromkeys(types, 1), []
    for n, t in zip(sizes, which):
        grads.append(flat[t][at[t]:at[t] + n])
        grads[-1].mul_(1.0 + len(grads) % 5)
        at[t] += n + 3
    return grads, flat


def _norms(torch, grads, kind):
    order = {"l2": 2.0, "l1": 1.0, "linf": math.inf}[kind]
    one = lambda t: torch.linalg.vector_norm(t, ord=order)  # noqa: E731
    norms = torch.stack([one(g.double()) if g.numel() else torch.zeros(
        (), dtype=torch.float64, device="cuda") for g in grads])
    return norms, one(norms)


@pytest.mark.parametrize("total", TOTALS + [PAST_THE_CACHES])
@pytest.mark.parametrize("types", ["mixed", "f32", "bf16"])
@pytest.mark.parametrize("kind", ["l2", "l1", "linf"])
def test_norms(total, types, kind):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(total % 1009)
    grads, _ = _grads(torch, total, types, gen)
    plan = ops.GradNorm(grads, norm=kind)
    plan.run()
    norms, common = _norms(torch, grads, kind)
    close = 0.0 if kind == "linf" else 1e-12
    assert bool(((plan.norms - norms).abs() <= close * norms).all())
    assert abs(float(plan.total) - float(common)) <= close * float(common)
    bits = plan.norms.clone(), plan.total.clone()
    # the same loaded for a clipping, and where the gradients then are
    assert torch.equal(plan.clip(math.inf), bits[1]) and torch.equal(plan.norms, bits[0])


@pytest.mark.parametrize("total", TOTALS + [PAST_THE_CACHES])
@pytest.mark.parametrize("types", ["mixed", "f32", "bf16"])
@pytest.mark.parametrize("out", [None, "float32", "bfloat16"])
def test_clip(total, types, out):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(total % 1009)
    grads, flat = _grads(torch, total, types, gen)
    before = {t: f.clone() for t, f in flat.items()}
    out_type = None if out is None else getattr(torch, out)
    outputs = None
    if out is not None:
        room = torch.full((total + 3 * len(grads) + 1,), 7.0, dtype=out_type, device="cuda")
        at, outputs = 1, []
        for g in grads:
            outputs.append(room[at:at + g.numel()])
            at += g.numel() + 3
    plan = ops.GradNorm(grads, outputs)
    total_norm = float(plan.clip(1.0, scale=-2.0))
    f = torch.tensor(-1.0 / total_norm, dtype=torch.float64).float().cuda()
    if out is None:
        # what lies between the tensors is as it was
        for t, old in before.items():
            want = old.clone()
            for g in grads:
                if g.dtype == t:
                    at = slice(g.storage_offset(), g.storage_offset() + g.numel())
                    want[at] = (old[at].float() * f).to(t)
            assert torch.equal(flat[t], want)
        return
    want = torch.full_like(room, 7.0)
    for g, o in zip(grads, outputs):
        want[o.storage_offset():o.storage_offset() + o.numel()] = (g.float() * f).to(out_type)
    assert torch.equal(room, want)
    assert all(torch.equal(flat[t], old) for t, old in before.items())


def test_what_each_call_writes():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    g = torch.tensor([3.0, 4.0], device="cuda")
    plan = ops.GradNorm([g, torch.full((1,), math.inf, device="cuda")])
    mark = lambda: (plan.norms.fill_(-1.0), plan.total.fill_(-1.0),  # noqa: E731
                    plan.found_nonfinite.fill_(-1))
    read = lambda: ([float(v) for v in plan.norms], float(plan.total),  # noqa: E731
                    int(plan.found_nonfinite))
    mark(), plan.run()
    assert read() == ([5.0, math.inf], math.inf, -1)
    mark(), plan.clip(1.0)
    assert read() == ([5.0, math.inf], math.inf, 1)
    mark(), plan.clip(1.0, total=torch.tensor(10.0, dtype=torch.float64, device="cuda"))
    assert read() == ([-1.0, -1.0], -1.0, 0)
    assert torch.equal(g, torch.tensor([3.0, 4.0], device="cuda") * torch.tensor(0.1).cuda())
