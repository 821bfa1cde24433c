"""The root-mean-square norm, its 8-bit form and its gradients against the formulas in 64
bits; how far fp32 may be off stands with the checks in rms_reference."""

import math

import pytest

import rms_reference as R
from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu

EPS = 1e-6
DIMS = [1, 2, 7, 8, 9, 63, 64, 65, 250, 511, 512, 513, 1000, 1024, 1025, 1600, 2048, 2049, 4096,
        4097, 8192, 8193, 16384, 16385, 40000, 65536]
FORWARD = [("bfloat16", None, "bfloat16", "bfloat16"),
           ("bfloat16", "bfloat16", "bfloat16", "bfloat16"),
           ("bfloat16", "float32", "float32", "bfloat16"), ("float32", "float32", None, "float32"),
           ("float32", None, "float32", "bfloat16"), ("bfloat16", None, None, "float32")]

TYPES = {"f": "float32", "h": "bfloat16", "-": None}
# rows, and the types of x, the result's gradient, the stream's and x's, the weight, and its
# gradient
GRADIENTS = [(1, *"fffff"), (7, *"hhhff"), (70, *"fhfhh"), (5, *"hff-f"), (33, *"ffhff"),
             (3, *"hhfff"), (2, *"hfh--"), (9, *"fhhf-")]


def _t(torch, name):
    return None if name is None else getattr(torch, name)


def _rows(torch, gen, tokens, dim, dtype, sigma=1.0):
    """Rows of different sizes with a few large columns."""
    t = torch.randn(tokens, dim, generator=gen, device="cuda")
    t *= torch.exp(2 * torch.rand(tokens, 1, generator=gen, device="cuda")) * sigma
    t[:, :: max(1, dim // 3)] *= 12.0
    return t.to(dtype)


def _case(torch, tokens, dim, x, res, weight, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(1000 * seed + 31 * tokens + dim)
    x = _rows(torch, gen, tokens, dim, _t(torch, x))
    res = None if res is None else _rows(torch, gen, tokens, dim, _t(torch, res), 3.0)
    w = None if weight is None else (1.0 + 0.3 * torch.randn(
        dim, generator=gen, device="cuda")).to(_t(torch, weight))
    return x, res, w, gen


def _sum(x, res):
    return x if res is None else (x.float() + res.float()).to(res.dtype)


@pytest.mark.parametrize("dim", DIMS)
def test_norm(dim):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    for tokens in (1, 3, 17):
        for k, (xt, rt, wt, ot) in enumerate(FORWARD):
            x, res, w, _ = _case(torch, tokens, dim, xt, rt, wt, k)
            got = ops.rms_norm(x, w, residual=res, eps=EPS, out_dtype=_t(torch, ot))
            h = _sum(x, res)
            if res is not None:
                got, summed = got
                assert torch.equal(summed, h)
            assert got.dtype == _t(torch, ot)
            R.check_norm(got, h, w, EPS)


@pytest.mark.parametrize("dim", DIMS)
def test_fp8(dim):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    for tokens, group in ((1, 0), (5, 32), (6, 64), (13, 128), (4, 256), (9, 0)):
        for k, (xt, rt, wt, _) in enumerate(FORWARD):
            x, res, w, _ = _case(torch, tokens, dim, xt, rt, wt, k)
            q, scales, *summed = ops.rms_norm_fp8(x, w, residual=res, eps=EPS, group=group)
            h = _sum(x, res)
            assert q.dtype == torch.float8_e4m3fn and q.shape == x.shape
            assert len(summed) == (res is not None)
            if summed:
                assert torch.equal(summed[0], h)
            R.check_fp8(q, scales, h, w, EPS, group)


@pytest.mark.parametrize("dim", DIMS)
def test_gradients(dim):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    for tokens, xt, yt, gt, wt, dwt in GRADIENTS:
        xt, yt, gt, wt, dwt = (TYPES[k] for k in (xt, yt, gt, wt, dwt))
        x, _, w, gen = _case(torch, tokens, dim, xt, None, wt)
        dy = _rows(torch, gen, tokens, dim, _t(torch, yt), 1e-3)
        for ds in (None, _rows(torch, gen, tokens, dim, _t(torch, gt), 1e-3)):
            gx = torch.full((tokens, dim), math.nan, dtype=_t(torch, gt), device="cuda")
            gw = None if dwt is None else torch.full((dim,), math.nan, dtype=_t(torch, dwt),
                                                     device="cuda")
            ops.rms_norm_grad(x, w, dy, gx, gw, eps=EPS, grad_sum=ds)
            R.check_grads(gx, gw, x, w, dy, ds, EPS)


@pytest.mark.parametrize("tokens,dim", [(4000, 64), (40000, 40), (9001, 1000), (5003, 1600),
                                        (3001, 4096), (700, 8192), (2000, 9000)])
def test_many_rows(tokens, dim):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    x, res, w, gen = _case(torch, tokens, dim, "bfloat16", "float32", "float32")
    out, h = ops.rms_norm(x, w, residual=res, eps=EPS)
    assert torch.equal(h, _sum(x, res))
    R.check_norm(out, h, w, EPS)
    q, scales, h2 = ops.rms_norm_fp8(x, w, residual=res, eps=EPS, group=128)
    assert torch.equal(h2, h)
    R.check_fp8(q, scales, h, w, EPS, 128)
    dy = _rows(torch, gen, tokens, dim, torch.bfloat16)
    ds = _rows(torch, gen, tokens, dim, torch.float32)
    gx = torch.empty_like(h)
    old = torch.randn(dim, generator=gen, device="cuda")
    gw = old.clone()
    ops.rms_norm_grad(h, w, dy, gx, gw, eps=EPS, grad_sum=ds, accumulate=True)
    R.check_grads(gx, gw, h, w, dy, ds, EPS, old)


def test_like_terms_do_not_stall():
    """2^17 rows alike: their sum's parts stay short."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    x = torch.full((1 << 17, 24), 1.1, device="cuda")
    dy = torch.full_like(x, 0.7)
    gw = torch.empty(24, device="cuda")
    ops.rms_norm_grad(x, None, dy, None, gw, eps=EPS)
    R.check_grads(None, gw, x, None, dy, None, EPS)


def test_gradient_against_differences():
    """Of sum(c * norm(x + t d) * w) at t = 0, in 64 bits by the formula, over a step whose
    third-order error is 1e-9 of it."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(5)
    for tokens, dim in ((1, 3), (6, 200), (4, 1500)):
        rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
        x, c, d = rand(tokens, dim), rand(tokens, dim), rand(tokens, dim)
        w, dw = rand(dim), rand(dim)
        value = lambda t: float((c.double() * R.norm(  # noqa: E731
            x.double() + t * d.double(), w.double() + t * dw.double(), EPS)[0]).sum())
        slope = (value(1e-4) - value(-1e-4)) / 2e-4
        gx, gw = torch.empty_like(x), torch.empty_like(w)
        ops.rms_norm_grad(x, w, c, gx, gw, eps=EPS)
        terms = torch.cat([(gx.double() * d).view(-1), gw.double() * dw])
        # the gradients' rounding (some 40 half steps of their terms) and the difference's
        assert abs(float(terms.sum()) - slope) <= 1e-5 * float(terms.abs().sum()) + 1e-6


def test_rows_of_zeros_infinities_and_nan():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    for dim in (5, 300, 3000):
        x, _, w, gen = _case(torch, 9, dim, "float32", None, "float32")
        x[1] = 0.0
        x[2, dim // 2] = math.inf
        x[3, 0] = math.nan
        x[4] = 1e30 * torch.randn(dim, generator=gen, device="cuda")  # squares pass fp32's range
        x[5] = 1e-30
        x[6, -1] = -math.inf
        R.check_norm(ops.rms_norm(x, w, eps=EPS), x, w, EPS)
        out = ops.rms_norm(x, w, eps=0.0)
        assert bool(out[1].isnan().all())
        keep = torch.tensor([0, 2, 3, 4, 5, 6, 7, 8], device="cuda")
        R.check_norm(out[keep], x[keep], w, 0.0)
        for group in (0, 32):
            q, scales = ops.rms_norm_fp8(x, w, eps=EPS, group=group)
            R.check_fp8(q, scales, x, w, EPS, group)
            assert not q[1].float().any() and bool((scales[1] == 2.0 ** -126).all())
        dy = torch.randn(9, dim, generator=gen, device="cuda")
        gx = torch.empty_like(x)
        ops.rms_norm_grad(x, w, dy, gx, eps=EPS)
        R.check_grads(gx, None, x, w, dy, None, EPS)
        # the rows beside them are as without them
        clean = x.clone()
        clean[2:4], clean[6] = 1.0, 1.0
        assert torch.equal(ops.rms_norm(clean, w, eps=EPS)[7:], ops.rms_norm(x, w, eps=EPS)[7:])


@pytest.mark.parametrize("dim", [6, 100, 700, 9000])
def test_rows_at_the_ends_of_fp32(dim):
    """Whose 1 / rms no fp32 number holds to its precision, or at all."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(dim)
    signs = torch.where(torch.rand(5, dim, generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    sizes = torch.tensor([3.3e38, 1e38, 1e-38, 1e-41, 2.0], device="cuda")[:, None]
    x = signs * sizes * (0.5 + 0.5 * torch.rand(5, dim, generator=gen, device="cuda"))
    w = torch.randn(dim, generator=gen, device="cuda")
    R.check_norm(ops.rms_norm(x, w, eps=0.0), x, w, 0.0)
    q, scales = ops.rms_norm_fp8(x, w, eps=0.0, group=32)
    R.check_fp8(q, scales, x, w, 0.0, 32)
    dy = torch.randn(5, dim, generator=gen, device="cuda")
    gx, gw = torch.empty_like(x), torch.empty_like(w)
    big = torch.tensor([0, 1, 4], device="cuda")  # the others' gradients pass fp32's range
    ops.rms_norm_grad(x[big], w, dy[big], gx[big], gw, eps=0.0)
    R.check_grads(None, gw, x[big], w, dy[big], None, 0.0)
    ops.rms_norm_grad(x, w, dy, None, gw, eps=0.0)
    R.check_grads(None, gw, x, w, dy, None, 0.0)


def test_an_infinite_weight():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    x, _, w, _ = _case(torch, 4, 100, "float32", None, "float32")
    w[40], w[41] = math.inf, math.nan
    R.check_norm(ops.rms_norm(x, w, eps=EPS), x, w, EPS)
    q, scales = ops.rms_norm_fp8(x, w, eps=EPS, group=32)
    assert bool(scales[:, 1].isnan().all()) and bool(q.float()[:, 32:64].isnan().all())
    assert bool(scales[:, [0, 2, 3]].isfinite().all())
    w[41] = 1.0
    q, scales = ops.rms_norm_fp8(x, w, eps=EPS, group=32)
    assert bool(scales[:, 1].isinf().all()) and bool(q.float()[:, 40].isnan().all())
    assert not q.float()[:, 32:40].any() and not q.float()[:, 41:64].any()


def test_no_rows():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    for dim in (40, 9000):
        x = torch.empty(0, dim, device="cuda")
        w = torch.ones(dim, device="cuda")
        assert ops.rms_norm(x, w).shape == (0, dim)
        out, summed = ops.rms_norm(x, w, residual=x)
        assert out.shape == summed.shape == (0, dim)
        q, scales, _ = ops.rms_norm_fp8(x, w, residual=x, group=32)
        assert q.shape == (0, dim) and scales.shape == (0, -(-dim // 32))
        gw = torch.full((dim,), 3.0, device="cuda")
        ops.rms_norm_grad(x, w, x, torch.empty_like(x), gw, grad_sum=x, accumulate=True)
        assert bool((gw == 3).all())
        ops.rms_norm_grad(x, w, x, torch.empty_like(x), gw)
        assert not gw.any()


@pytest.mark.parametrize("dim", [64, 61, 1600, 9000])
def test_slices_of_wider_buffers(dim):
    """Rows that lie between others', at any element, and results between them."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(dim)
    for dtype in (torch.float32, torch.bfloat16):
        wide = torch.randn(21, 4 * dim + 7, generator=gen, device="cuda").to(dtype)
        before = wide.clone()
        x, res = wide[:, 1:dim + 1], wide[:, dim + 2:2 * dim + 2]
        out, summed = wide[:, 2 * dim + 3:3 * dim + 3], wide[:, 3 * dim + 4:4 * dim + 4]
        w = torch.randn(dim + 1, generator=gen, device="cuda").to(dtype)[1:]
        h = _sum(x, res)
        ops.rms_norm(x, w, residual=res, eps=EPS, out=out, summed=summed)
        assert torch.equal(summed, h)
        R.check_norm(out, h, w, EPS)
        kept = torch.ones(4 * dim + 7, dtype=torch.bool, device="cuda")
        kept[2 * dim + 3:3 * dim + 3] = kept[3 * dim + 4:4 * dim + 4] = False
        assert torch.equal(wide[:, kept], before[:, kept])
        dy, gx = x, wide[:, 2 * dim + 3:3 * dim + 3]
        gw = torch.zeros(dim, dtype=dtype, device="cuda")
        ops.rms_norm_grad(h, w, dy, gx, gw, eps=EPS, grad_sum=res)
        R.check_grads(gx, gw, h, w, dy, res, EPS)
        assert torch.equal(wide[:, kept], before[:, kept])
        bytes_ = torch.zeros(21, 2 * dim + 3, dtype=torch.uint8, device="cuda")
        q = bytes_.view(torch.float8_e4m3fn)[:, 1:dim + 1]
        _, scales = ops.rms_norm_fp8(x, w, eps=EPS, group=64, out=q)
        R.check_fp8(q, scales, x, w, EPS, 64)
        assert not bytes_[:, 0].any() and not bytes_[:, dim + 1:].any()


@pytest.mark.parametrize("dim", [100, 1600, 9001])
def test_in_place(dim):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    x, res, w, gen = _case(torch, 50, dim, "bfloat16", "bfloat16", "bfloat16")
    want, total = ops.rms_norm(x, w, residual=res, eps=EPS)
    a, b = x.clone(), res.clone()
    got = ops.rms_norm(a, w, residual=b, eps=EPS, out=a, summed=b)
    assert got[0] is a and got[1] is b and torch.equal(a, want) and torch.equal(b, total)
    a, b = x.clone(), res.clone()
    ops.rms_norm(a, w, residual=b, eps=EPS, out=b, summed=a)
    assert torch.equal(b, want) and torch.equal(a, total)
    a = x.clone()
    ops.rms_norm(a, w, residual=a, eps=EPS, out=a)  # twice x
    R.check_norm(a, (x.float() * 2).bfloat16(), w, EPS)
    b = res.clone()
    q, scales = ops.rms_norm_fp8(x, w, residual=b, eps=EPS, summed=b)[:2]
    assert torch.equal(b, total)
    R.check_fp8(q, scales, total, w, EPS, 0)
    dy, ds = _rows(torch, gen, 50, dim, x.dtype), _rows(torch, gen, 50, dim, x.dtype)
    gx, gw = torch.empty_like(x), torch.empty_like(w)
    ops.rms_norm_grad(x, w, dy, gx, gw, eps=EPS, grad_sum=ds)
    for k in range(3):
        t = [x.clone(), dy.clone(), ds.clone()]
        w2 = torch.empty_like(w)
        ops.rms_norm_grad(t[0], w, t[1], t[k], w2, eps=EPS, grad_sum=t[2])
        assert torch.equal(t[k], gx) and torch.equal(w2, gw)


def test_same_bits_twice_on_a_stream_and_in_a_graph():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    for tokens, dim in ((3, 200), (2500, 1000), (300, 9000)):
        x, res, w, gen = _case(torch, tokens, dim, "bfloat16", "float32", "float32")
        dy = _rows(torch, gen, tokens, dim, torch.bfloat16)
        gw = torch.empty_like(w)
        gx = torch.empty_like(res)

        def call():
            out, h = ops.rms_norm(x, w, residual=res, eps=EPS)
            q, scales = ops.rms_norm_fp8(x, w, eps=EPS, group=64)
            ops.rms_norm_grad(h, w, dy, gx, gw, eps=EPS, grad_sum=res)
            return out, h, q.view(torch.uint8), scales

        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = call()
        side = torch.cuda.Stream()
        for k in range(3):
            x.copy_(_rows(torch, gen, tokens, dim, torch.bfloat16))
            graph.replay()
            torch.cuda.synchronize()
            first = [t.clone() for t in (*held, gx, gw)]
            gx.zero_(), gw.zero_()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                again = call()
            torch.cuda.synchronize()
            for a, b in zip(first, (*again, gx, gw)):
                assert torch.equal(a, b), k


def test_rows_past_one_axis_of_workgroups():
    """More workgroups than one axis of a launch has in this library."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    tokens = (1 << 23) + 5
    x = torch.ones(tokens, 8, dtype=torch.bfloat16, device="cuda")
    x[-1] = 2.0
    x[-1, 0] = 0.0
    out = ops.rms_norm(x, eps=0.0)
    assert bool((out[:-1] == 1).all())
    R.check_norm(out[-1:], x[-1:], None, 0.0)
    gx, gw = torch.empty_like(x), torch.empty(8, device="cuda")
    ops.rms_norm_grad(x, None, x, gx, gw, eps=0.0)
    # a row's own direction has no gradient; the sums are of ones, and the last row's
    assert float(gx.float().abs().max()) <= 2.0 ** -20
    want = torch.full((8,), tokens - 1.0, dtype=torch.float64)
    want[1:] += 2.0 * math.sqrt(8 / 7)
    assert bool(((gw.double().cpu() - want).abs() <= want * 4 * R.ULP).all())


def test_offsets_past_32_bits():
    """Rows whose elements lie beyond 2^32 from the first."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    tokens, dim = 70000, 1 << 16
    x = torch.zeros(tokens, dim, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(0)
    at = torch.tensor([0, 32768, 65535, 65536, 65537, tokens - 1], device="cuda")
    x[at] = torch.randn(len(at), dim, generator=gen, device="cuda").bfloat16()
    out = ops.rms_norm(x, eps=EPS)
    R.check_norm(out[at], x[at], None, EPS)
    assert not out[1].any() and not out[65538].any()
    gw = torch.empty(dim, device="cuda")
    ops.rms_norm_grad(x, None, x, out, gw, eps=EPS, grad_sum=x)
    R.check_grads(out[at], gw, x[at], None, x[at], x[at], EPS)


def test_refusals():
    torch = torch_cuda()
    from paper_1904_00962_amd import _lib, ops
    x = torch.zeros(4, 16, device="cuda")
    w = torch.ones(16, device="cuda")
    half = x.bfloat16()
    for call in (lambda: ops.rms_norm(x.half()), lambda: ops.rms_norm(x, w.half()),
                 lambda: ops.rms_norm(x, residual=x.half()),
                 lambda: ops.rms_norm(x, out_dtype=torch.float16),
                 lambda: ops.rms_norm(x, out=half, out_dtype=torch.float32),
                 lambda: ops.rms_norm(x, residual=x.clone(), summed=half),
                 lambda: ops.rms_norm_fp8(x, out=x),
                 lambda: ops.rms_norm_fp8(x, scales=torch.zeros(4, 1, device="cuda").bfloat16()),
                 lambda: ops.rms_norm_grad(x, w, x.half(), x),
                 lambda: ops.rms_norm_grad(x, w, x, x.half()),
                 lambda: ops.rms_norm_grad(x, w, x, half, grad_sum=x),
                 lambda: ops.rms_norm_grad(x, w, x, None, w.half())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ops.rms_norm(x.cpu()), lambda: ops.rms_norm(x, w.cpu()),
                 lambda: ops.rms_norm(x[0]), lambda: ops.rms_norm(x.t()),
                 lambda: ops.rms_norm(x, w[:8]),
                 lambda: ops.rms_norm(x, torch.ones(32, device="cuda")[::2]),
                 lambda: ops.rms_norm(x, residual=x[:3]), lambda: ops.rms_norm(x, summed=x.clone()),
                 lambda: ops.rms_norm(x, out=x[:3]),
                 lambda: ops.rms_norm_fp8(x, scales=torch.zeros(4, 2, device="cuda")),
                 lambda: ops.rms_norm_grad(x, w, x[:3]), lambda: ops.rms_norm_grad(x, w, x, x[:2]),
                 lambda: ops.rms_norm_grad(x, w, x, None, grad_sum=x),
                 lambda: ops.rms_norm_grad(x, w, x, None, w[:4]),
                 lambda: ops.rms_norm(x.clone().requires_grad_())):
        with pytest.raises(ValueError):
            call()
    with torch.no_grad():
        ops.rms_norm(x.clone().requires_grad_())
    for status, call in ((_lib.LAMB_EINVAL, lambda: ops.rms_norm(x, eps=-1.0)),
                         (_lib.LAMB_EINVAL, lambda: ops.rms_norm(x, eps=math.nan)),
                         (_lib.LAMB_EINVAL, lambda: ops.rms_norm(x, residual=half)),
                         (_lib.LAMB_EINVAL, lambda: ops.rms_norm_fp8(x, group=48)),
                         (_lib.LAMB_EINVAL, lambda: ops.rms_norm_fp8(x, group=-32)),
                         (_lib.LAMB_EOVERLAP, lambda: ops.rms_norm(x[1:], out=x[:3])),
                         (_lib.LAMB_EOVERLAP, lambda: ops.rms_norm(x, x[0], out=x)),
                         (_lib.LAMB_EOVERLAP, lambda: ops.rms_norm(
                             half, out=x.view(torch.bfloat16).view(4, 32)[:, :16], residual=x)),
                         (_lib.LAMB_EOVERLAP, lambda: ops.rms_norm_grad(x, w, x.clone(), x, w))):
        with pytest.raises(_lib.LambError) as e:
            call()
        assert e.value.status == status
