"""Plain 64-bit evaluations of the root-mean-square norm, its gradients and its 8-bit form,
with how far fp32 arithmetic may be off, that the tests compare the kernels with."""

import torch

ULP = 2.0 ** -24  # half a step of fp32, relative to the value
TINY = 2.0 ** -126  # below it a type's own steps stop shrinking


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def norm(h, weight, eps):
    """(y in 64 bits, r) for the rows of h."""
    h = h.double()
    r = 1.0 / torch.sqrt((h * h).mean(dim=1, keepdim=True) + eps)
    y = h * r
    return (y if weight is None else y * weight.double()), r


def check_norm(got, h, weight, eps):
    """r is rounded to fp32 once, and each of the two products (the sums are in fp64, the
    quotient and the root of them at most 2^-50 off); then the result to its type."""
    want, _ = norm(h, weight, eps)
    bound = want.abs() * (4 * ULP + half_step(got.dtype) * (1 + 4 * ULP)) + TINY
    ok = _same_where_not_finite(got, want)
    off = (got.double() - want).abs()
    assert bool((off[ok] <= bound[ok]).all()), float((off / bound)[ok].max())


def _same_where_not_finite(got, want):
    """Where ``want`` is finite; the NaN and infinities of both are the same."""
    assert torch.equal(got.isnan(), want.isnan())
    infinite = want.isinf()
    assert torch.equal(got.double()[infinite], want[infinite])
    return want.isfinite()


def check_fp8(q, scales, h, weight, eps, group):
    """A scale is off by fp32's roundings: three of y and one of the division. A value, with
    its scale, is off by half a step of e4m3 (2^-4 of it, or 2^-10 scales where it is below
    2^-6 scales), by y's three roundings and the division's."""
    want, _ = norm(h, weight, eps)
    n, d = want.shape
    group = group or d
    parts = torch.nn.functional.pad(want, (0, -d % group)).view(n, -1, group)
    top = parts.abs().amax(dim=2)  # NaN where a group holds one
    scale = (top / 448.0).clamp(min=2.0 ** -126)
    assert scales.shape == scale.shape and scales.dtype == torch.float32
    assert torch.equal(scales.isnan(), scale.isnan())
    ok = scale.isfinite()
    assert bool(((scales.double() - scale).abs()[ok] <= scale[ok] * 5 * ULP).all())
    each = scales.double().repeat_interleave(group, dim=1)[:, :d]
    ok = ok.repeat_interleave(group, dim=1)[:, :d]
    assert bool(q.float()[each.isnan()].isnan().all())
    off = (q.double() * each - want).abs()
    bound = torch.maximum(want.abs() * 2.0 ** -4, each * 2.0 ** -10) * (1 + 8 * ULP) \
        + want.abs() * 6 * ULP
    assert bool((off[ok] <= bound[ok]).all()), float((off / bound)[ok].max())
    largest = torch.nn.functional.pad(q.float(), (0, -d % group)).view(n, -1, group).abs()
    full = scale.isfinite() & (top >= 448.0 * 2.0 ** -126)
    assert bool((largest.amax(dim=2)[full] == 448).all())


def grads(h, weight, dy, ds, eps):
    """(dh, dw, bound of dh's error in fp32 before its own rounding, size of dw's terms)."""
    h, dy = h.double(), dy.double()
    w = torch.ones(h.shape[1], dtype=torch.float64, device=h.device) if weight is None \
        else weight.double()
    r = 1.0 / torch.sqrt((h * h).mean(dim=1, keepdim=True) + eps)
    x = h * r
    g = dy * w
    mean = (g * x).mean(dim=1, keepdim=True)
    mean_size = (g * x).abs().mean(dim=1, keepdim=True)
    dh = r * (g - x * mean)
    # g: one rounding; x: two (r, the product); the mean: g's, in the sum, and its own; then
    # two fused products, each rounded once, and r's rounding again
    bound = ULP * (r * (g.abs() + x.abs() * (mean_size + 3 * mean.abs())) + 2 * dh.abs())
    if ds is not None:
        dh = dh + ds.double()
    bound = 1.01 * (bound + ULP * dh.abs())
    terms = dy * x
    return dh, terms.sum(dim=0), bound, terms.abs().sum(dim=0)


def check_grads(grad_x, grad_weight, h, weight, dy, ds, eps, old=None):
    dh, dw, bound, size = grads(h, weight, dy, ds, eps)
    if grad_x is not None:
        limit = bound + half_step(grad_x.dtype) * (dh.abs() + bound) + TINY
        off = (grad_x.double() - dh).abs()
        ok = _same_where_not_finite(grad_x, dh)
        assert bool((off[ok] <= limit[ok]).all()), float((off / limit)[ok].max())
    if grad_weight is not None:
        # a term has two roundings (x's), a sum in fp32 one for each of 32 terms and of the
        # sums of 32; the join is in fp64
        folds = h.shape[0] / (32 * 256) + 1
        error = size * ULP * (2 + 32 + folds)
        want = dw if old is None else dw + old.double()
        limit = error + half_step(grad_weight.dtype) * (want.abs() + error) + TINY
        off = (grad_weight.double() - want).abs()
        assert bool((off <= limit).all()), float((off / limit).max())
