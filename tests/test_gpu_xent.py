"""Cross entropy against a vocabulary table, and its gradients, against the formulas in
64 bits.

Tolerances. Logits are sums of exact products in fp32: off by at most dim 2^-24 of the
sum of magnitudes, in practice by far less; losses are held to 2e-6 (1 + largest
logit). Q is rounded to bf16, and so is a bf16 result, each entry by at most 2^-8 and
by 2^-9.2 in the root mean square: the gradients are held, as a 2-norm, to 2^-8 (the
two together are 2^-8.7) of the sums of magnitudes of their terms, which the fp32
errors of lse stay below."""

import math

import pytest

import ops_reference as R
from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu

GRAD = 2.0 ** -8


def _problem(torch, tokens, dim, vocab, seed=0, spread=1.0, ignored=0.0, dtype=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn(tokens, dim, generator=gen, device="cuda").mul_(spread).to(torch.bfloat16)
    w = torch.randn(vocab, dim, generator=gen, device="cuda").mul_(0.1).to(torch.bfloat16)
    t = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
    t[torch.rand(tokens, generator=gen, device="cuda") < ignored] = -100
    return h, w, t.to(dtype or torch.int64)


def _check(torch, h, w, t, out_dtype=None, **kw):
    from paper_1904_00962_amd import ops
    mean, loss, lse = ops.linear_cross_entropy(h, w, t)
    gh = torch.full(h.shape, math.nan, dtype=torch.bfloat16, device="cuda")
    gw = torch.full(w.shape, math.nan, dtype=out_dtype or torch.bfloat16, device="cuda")
    ops.linear_cross_entropy_grad(h, w, t, lse, gh, gw, **kw)
    r_mean, r_loss, r_gh, r_gw, s_gh, s_gw = R.cross_entropy(
        h, w, t, reduction=kw.get("reduction", "mean"))
    big = float((h.double() @ w.double().t().contiguous()).abs().max()) if h.numel() else 0.0
    assert float((loss.double() - r_loss).abs().max() if len(t) else 0) <= 2e-6 * (1 + big)
    assert abs(float(mean) - float(r_mean)) <= 2e-6 * (1 + big)
    for got, want, size in ((gh, r_gh, s_gh), (gw, r_gw, s_gw)):
        off = float(torch.linalg.vector_norm(got.double() - want))
        assert off <= GRAD * float(torch.linalg.vector_norm(size)) + 1e-12


@pytest.mark.parametrize("tokens", [1, 2, 63, 64, 65, 129, 700])
@pytest.mark.parametrize("dim,vocab", [(8, 1), (64, 5), (33, 127), (100, 1000), (256, 2003),
                                       (1, 300), (72, 257)])
def test_sizes(tokens, dim, vocab):
    torch = torch_cuda()
    _check(torch, *_problem(torch, tokens, dim, vocab, seed=tokens + dim))


@pytest.mark.parametrize("tokens,dim,vocab", [(1200, 256, 30522), (3000, 200, 9000),
                                              (5000, 64, 50257)])
@pytest.mark.parametrize("out", ["bfloat16", "float32"])
def test_larger_tiles_and_several_pieces(tokens, dim, vocab, out):
    torch = torch_cuda()
    _check(torch, *_problem(torch, tokens, dim, vocab, ignored=0.1), getattr(torch, out))


@pytest.mark.parametrize("ignored", [0.3, 0.9, 1.0])
def test_ignored_tokens_reach_nothing(ignored):
    """Their rows hold NaN and infinities; only the others' results are left."""
    torch = torch_cuda()
    h, w, t = _problem(torch, 500, 96, 777, ignored=ignored, dtype=torch.int32)
    clean = h.clone()
    gone = (t == -100).nonzero()[:, 0]
    h[gone[::2]] = math.nan
    h[gone[1::2]] = math.inf
    from paper_1904_00962_amd import ops
    mean, loss, lse = ops.linear_cross_entropy(h, w, t)
    gh, gw = torch.full_like(h, 7.0), torch.full_like(w, 7.0)
    ops.linear_cross_entropy_grad(h, w, t, lse, gh, gw)
    m2, l2, lse2 = ops.linear_cross_entropy(clean, w, t)
    gh2, gw2 = torch.full_like(h, 7.0), torch.full_like(w, 7.0)
    ops.linear_cross_entropy_grad(clean, w, t, lse2, gh2, gw2)
    assert torch.equal(mean, m2) and torch.equal(loss, l2)
    assert torch.equal(gh, gh2) and torch.equal(gw, gw2)
    assert not gh[gone].any() and not loss[gone].any()
    if ignored == 1.0:
        assert float(mean) == 0.0 and not gw.any()
    _check(torch, clean, w, t)


def test_no_tokens():
    torch = torch_cuda()
    h, w, t = _problem(torch, 0, 16, 50)
    _check(torch, h, w, t)


def test_reductions_upstream_gradients_and_accumulation():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    h, w, t = _problem(torch, 150, 64, 900, ignored=0.2)
    _check(torch, h, w, t, reduction="sum")
    _, _, lse = ops.linear_cross_entropy(h, w, t)
    _, _, r_gh, r_gw, s_gh, s_gw = (R.cross_entropy(h, w, t))[0:6]
    gh = torch.empty_like(h)
    up = torch.tensor([3.0], device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        gw = torch.full(w.shape, 0.25, dtype=dtype, device="cuda")
        ops.linear_cross_entropy_grad(h, w, t, lse, gh, gw, grad_loss=up, grad_scale=0.5,
                                      accumulate=True)
        size = 1.5 * float(torch.linalg.vector_norm(s_gw)) + 0.25 * math.sqrt(gw.numel())
        assert float(torch.linalg.vector_norm(gw.double() - 0.25 - 1.5 * r_gw)) <= GRAD * size
        assert float(torch.linalg.vector_norm(gh.double() - 1.5 * r_gh)) <= \
            GRAD * 1.5 * float(torch.linalg.vector_norm(s_gh))
    only = torch.empty_like(h)
    ops.linear_cross_entropy_grad(h, w, t, lse, only, None, grad_loss=up, grad_scale=0.5)
    assert torch.equal(only, gh)
    one, both = torch.empty_like(w), torch.empty_like(w)
    ops.linear_cross_entropy_grad(h, w, t, lse, None, one)
    ops.linear_cross_entropy_grad(h, w, t, lse, gh, both)
    assert torch.equal(one, both)


def test_strides_and_alignment():
    """Rows at odd addresses and of any stride, in and out; nothing beside is written."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    h, w, t = _problem(torch, 130, 72, 333)
    wide_h = torch.zeros(130, 200, dtype=torch.bfloat16, device="cuda")
    wide_w = torch.zeros(333, 101, dtype=torch.bfloat16, device="cuda")
    vh, vw = wide_h[:, 3:75], wide_w[:, 5:77]
    vh.copy_(h)
    vw.copy_(w)
    mean, loss, lse = ops.linear_cross_entropy(h, w, t)
    m2, l2, lse2 = ops.linear_cross_entropy(vh, vw, t)
    assert torch.equal(loss, l2) and torch.equal(lse, lse2) and torch.equal(mean, m2)
    gh, gw = torch.empty_like(h), torch.empty_like(w)
    ops.linear_cross_entropy_grad(h, w, t, lse, gh, gw)
    oh = torch.full((130, 90), 7.0, dtype=torch.bfloat16, device="cuda")
    ow = torch.full((333, 85), 7.0, dtype=torch.bfloat16, device="cuda")
    ops.linear_cross_entropy_grad(vh, vw, t, lse, oh[:, 1:73], ow[:, 7:79])
    assert torch.equal(oh[:, 1:73], gh) and torch.equal(ow[:, 7:79], gw)
    for o, a, b in ((oh, 1, 73), (ow, 7, 79)):
        assert bool((o[:, :a] == 7).all()) and bool((o[:, b:] == 7).all())
    # a strided table that can be read in place
    big = torch.zeros(333, 128, dtype=torch.bfloat16, device="cuda")
    big[:, :72].copy_(w)
    m3, l3, _ = ops.linear_cross_entropy(h, big[:, :72], t)
    assert torch.equal(l3, loss) and torch.equal(m3, mean)


def test_large_logits_and_nonfinite_values():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    _check(torch, *_problem(torch, 100, 64, 500, spread=300.0))  # logits in the hundreds
    h, w, t = _problem(torch, 40, 32, 200)
    want = ops.linear_cross_entropy(h, w, t)[1]
    bad = h.clone()
    bad[7, 3] = math.nan
    mean, loss, _ = ops.linear_cross_entropy(bad, w, t)
    rest = torch.arange(40, device="cuda") != 7
    assert math.isnan(float(loss[7])) and math.isnan(float(mean))
    assert torch.equal(loss[rest], want[rest])
    # a word that cannot come: its logit is -inf for every token (hidden all positive)
    w2, h2 = w.clone(), h.abs() + 0.125
    w2[11] = -math.inf
    t2 = torch.where(t == 11, 12, t)
    _, loss, _ = ops.linear_cross_entropy(h2, w2, t2)
    keep = [v for v in range(200) if v != 11]
    index = torch.tensor([keep.index(int(v)) for v in t2], device="cuda")
    r = R.cross_entropy(h2, w[keep], index)[1]
    assert float((loss.double() - r).abs().max()) < 1e-5


def test_a_target_outside_the_vocabulary_shows():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    h, w, t = _problem(torch, 70, 32, 90)
    for bad in (90, -1, 2 ** 40):
        t2 = t.clone()
        t2[5] = bad
        mean, loss, lse = ops.linear_cross_entropy(h, w, t2)
        assert math.isnan(float(mean)) and math.isnan(float(loss[5]))
        assert int(loss.isnan().sum()) == 1
        gh, gw = torch.empty_like(h), torch.empty_like(w)
        ops.linear_cross_entropy_grad(h, w, t2, lse, gh, gw)
        assert gh[5].isnan().all() and gw.isnan().all() and not gh[:5].isnan().any()


def test_gradient_against_differences():
    """Along a direction, the mean's difference quotient, with table and hidden moved by
    bf16 values of one exponent so that the moved points are exact."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    h, w, t = _problem(torch, 64, 48, 300, ignored=0.1)
    # values on a grid of 2^-6, so that a step of 2^-6 stays a bf16 value
    h, w = ((x.float() * 64).round().clamp(-100, 100) / 64 for x in (h, w))
    gen = torch.Generator(device="cuda").manual_seed(2)
    dh, dw = (torch.randint(-1, 2, x.shape, generator=gen, device="cuda").float() / 64
              for x in (h, w))
    f = lambda k: R.cross_entropy(h + k * dh, w + k * dw, t)[0]  # noqa: E731
    slope = float((8 * (f(1) - f(-1)) - (f(2) - f(-2))) / 12)
    hb, wb = h.bfloat16(), w.bfloat16()
    assert torch.equal(hb.float(), h) and torch.equal(wb.float(), w)
    _, _, lse = ops.linear_cross_entropy(hb, wb, t)
    gh, gw = torch.empty_like(hb), torch.empty(w.shape, device="cuda")
    ops.linear_cross_entropy_grad(hb, wb, t, lse, gh, gw)
    got = float((gh.double() * dh).sum() + (gw.double() * dw).sum())
    size = float((gh.double() * dh).abs().sum() + (gw.double() * dw).abs().sum())
    assert abs(got - slope) <= GRAD * size


def test_same_bits_twice_and_in_a_graph():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    h, w, t = _problem(torch, 333, 64, 3000, ignored=0.2)
    gh, gw = torch.empty_like(h), torch.empty_like(w)

    def call():
        out = ops.linear_cross_entropy(h, w, t)
        ops.linear_cross_entropy_grad(h, w, t, out[2], gh, gw)
        return out

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for k in range(3):
        h2, _, t2 = _problem(torch, 333, 64, 3000, seed=k + 1, ignored=0.3 * k)
        h.copy_(h2)
        t.copy_(t2)
        graph.replay()
        torch.cuda.synchronize()
        first = [x.clone() for x in (*held, gh, gw)]
        again = call()
        torch.cuda.synchronize()
        for a, b in zip(first, (*again, gh, gw)):
            assert torch.equal(a, b), k


def test_refusals():
    torch = torch_cuda()
    from paper_1904_00962_amd import _lib, ops
    h, w, t = _problem(torch, 10, 16, 20)
    for bad in ((h.float(), w, t), (h, w.float(), t), (h, w, t.float())):
        with pytest.raises(TypeError):
            ops.linear_cross_entropy(*bad)
    for bad in ((h[:, :8], w, t), (h, w, t[:5]), (h.cpu(), w, t), (h.t().contiguous().t(), w, t),
                (h, w, t[::2])):
        with pytest.raises(ValueError):
            ops.linear_cross_entropy(*bad)
    _, _, lse = ops.linear_cross_entropy(h, w, t)
    with pytest.raises(ValueError):
        ops.linear_cross_entropy_grad(h, w, t, lse, h[:5])
    with pytest.raises(_lib.LambError) as e:  # a gradient over its own input
        ops.linear_cross_entropy_grad(h, w, t, lse, h)
    assert e.value.status == _lib.LAMB_EOVERLAP
    with pytest.raises(ValueError):
        ops.linear_cross_entropy_grad(h, w, t, lse, reduction="none")


def _sampled_lse(torch, h, w, rows):
    return torch.logsumexp(h[rows].double().cpu() @ w.double().cpu().t(), dim=1)


def test_many_tokens_and_words():
    """More workgroups than a launch takes along one axis, several groups of tokens packed
    by each, and parts past 2^32 bytes."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    tokens, dim, vocab = 1 << 22, 8, 1 << 18
    h, w, t = _problem(torch, tokens, dim, vocab, ignored=0.25)
    mean, loss, lse = ops.linear_cross_entropy(h, w, t)
    keep = t != -100
    rows = torch.nonzero(keep)[:, 0]
    rows = torch.cat([rows[:40], rows[len(rows) // 2:][:40], rows[-40:]])
    want = _sampled_lse(torch, h, w, rows)
    mine = (h[rows].double() * w[t[rows]].double()).sum(1).cpu()
    assert float((lse[rows].cpu().double() - want).abs().max()) < 4e-5
    assert float((loss[rows].cpu().double() - (want - mine)).abs().max()) < 4e-5
    assert bool(loss[~keep].eq(0).all()) and bool(loss[keep].gt(0).all())
    assert abs(float(mean) - float(loss.double().sum() / keep.sum())) < 1e-5


def test_gradient_of_the_most_tokens():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    tokens, dim, vocab = 1 << 24, 8, 8
    h, w, t = _problem(torch, tokens, dim, vocab, ignored=0.25)
    logits = h.float() @ w.float().t().contiguous()
    lse = torch.logsumexp(logits, dim=1)
    gh = torch.full_like(h, math.nan)
    gw = torch.full(w.shape, math.nan, device="cuda")
    ops.linear_cross_entropy_grad(h, w, t, lse, gh, gw, reduction="sum")
    q = torch.exp(logits - lse[:, None])
    q.scatter_add_(1, t.clamp(min=0)[:, None], torch.full((tokens, 1), -1.0, device="cuda"))
    q.mul_((t != -100)[:, None])
    want = q @ w.float()
    size = q.abs() @ w.float().abs()
    assert bool(((gh.float() - want).abs() <= 2 * GRAD * size + 1e-6).all())
    assert bool(gh[t == -100].eq(0).all())
    q, size = q.t().contiguous(), q.abs().t().contiguous()
    off = float(torch.linalg.vector_norm(gw - q @ h.float()))
    assert off <= GRAD * float(torch.linalg.vector_norm(size @ h.float().abs()))
