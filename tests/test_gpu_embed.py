"""The token table's lookup and gradient against the formulas in 64 bits.

Tolerances. A looked-up value is a product in fp32, rounded once more to its type: it
is compared with exactly that. A gradient is a sum of n terms in fp32 (off by at most
n 2^-24 of the sum of magnitudes), rounded to its type (half a unit of bf16's last place)."""

import math

import pytest

from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu


def _reference(torch, ids, rows, vocab, scale, skip=None):
    ids = ids.reshape(-1).long()
    keep = (ids >= 0) & (ids < vocab)
    if skip is not None:
        keep &= ids != skip
    sums = torch.zeros(vocab, rows.shape[1], dtype=torch.float64, device="cuda")
    size, count = torch.zeros_like(sums), torch.zeros(vocab, dtype=torch.float64, device="cuda")
    r = rows.double()[keep] * scale
    sums.index_add_(0, ids[keep], r)
    size.index_add_(0, ids[keep], r.abs())
    count.index_add_(0, ids[keep], torch.ones(len(r), dtype=torch.float64, device="cuda"))
    return sums, size, count


def _ids(torch, kind, tokens, vocab, gen, dtype):
    if kind == "uniform":
        t = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
    elif kind == "text":  # the k-th id 1 / k as frequent
        u = torch.rand(tokens, generator=gen, device="cuda")
        t = (torch.exp(u * math.log(vocab + 1.0)) - 1).long().clamp(0, vocab - 1)
        t = torch.randperm(vocab, generator=gen, device="cuda")[t]
    elif kind == "one":
        t = torch.full((tokens,), vocab - 1, device="cuda")
    else:  # sorted runs around the lengths where a chunk ends
        t = torch.arange(tokens, device="cuda") // 33 % vocab
    return t.to(dtype)


def _check_grad(torch, ids, rows, out, vocab, scale, old=None, skip=None):
    sums, size, count = _reference(torch, ids, rows, vocab, scale, skip)
    want = sums if old is None else old.double() + sums
    size = size + (0 if old is None else old.double().abs())
    bound = size * (count[:, None] + 4) * 2.0 ** -24
    if out.dtype == torch.bfloat16:
        # bound so far may carry the sum over a power of two
        binade = torch.exp2(torch.floor(torch.log2(want.abs() + bound + 1e-300)))
        bound = bound + binade * 2.0 ** -8
    assert bool(((out.double() - want).abs() <= bound + 1e-30).all())
    if old is not None:
        assert torch.equal(out[count == 0], old[count == 0])


@pytest.mark.parametrize("kind", ["uniform", "text", "one", "runs"])
@pytest.mark.parametrize("tokens,dim,vocab", [(1, 1, 1), (3, 8, 2), (31, 24, 7), (32, 513, 64),
                                              (33, 40, 65), (64, 64, 1000), (1000, 100, 300),
                                              (2100, 1030, 129), (5000, 16, 50257)])
def test_gradients(kind, tokens, dim, vocab):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(tokens + dim)
    for r_dtype, t_dtype, i_dtype in ((torch.float32, torch.float32, torch.int64),
                                      (torch.bfloat16, torch.bfloat16, torch.int32),
                                      (torch.bfloat16, torch.float32, torch.int64)):
        ids = _ids(torch, kind, tokens, vocab, gen, i_dtype)
        rows = torch.randn(tokens, dim, generator=gen, device="cuda").to(r_dtype)
        out = torch.full((vocab, dim), math.nan, dtype=t_dtype, device="cuda")
        ops.embedding_grad(ids, rows, out, scale=1.5)
        _check_grad(torch, ids, rows, out, vocab, 1.5)
        old = torch.randn(vocab, dim, generator=gen, device="cuda").to(t_dtype)
        out = old.clone()
        ops.embedding_grad(ids, rows, out, scale=0.5, accumulate=True)
        _check_grad(torch, ids, rows, out, vocab, 0.5, old)


@pytest.mark.parametrize("tokens", [40000, 300000])
def test_many_tokens(tokens):
    """Ranges of ids get wider where tokens are many."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids = _ids(torch, "text", tokens, 3001, gen, torch.int64)
    rows = torch.randn(tokens, 16, generator=gen, device="cuda")
    out = torch.empty(3001, 16, device="cuda")
    ops.embedding_grad(ids, rows, out)
    _check_grad(torch, ids, rows, out, 3001, 1.0)


def test_padding_and_ids_outside_the_table():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(4)
    ids = _ids(torch, "text", 900, 50, gen, torch.int64)
    ids[::7] = 3
    ids[5], ids[6], ids[899] = -1, 50, 2 ** 40
    rows = torch.randn(900, 72, generator=gen, device="cuda")
    rows[ids == 3] = math.nan  # a padding token's gradient is not looked at
    rows[5] = math.inf
    out = torch.empty(50, 72, device="cuda")
    ops.embedding_grad(ids, rows, out, padding_id=3)
    _check_grad(torch, ids, torch.where((ids == 3)[:, None], 0.0, rows), out, 50, 1.0, skip=3)
    assert not out[3].any()
    table = torch.randn(50, 72, generator=gen, device="cuda")
    got = ops.embedding(ids, table, scale=2.0)
    bad = (ids < 0) | (ids >= 50)
    assert got[bad].isnan().all() and int(bad.sum()) == 3
    assert torch.equal(got[~bad], table[ids[~bad]] * 2.0)


def test_no_tokens():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    table = torch.ones(5, 8, device="cuda")
    assert ops.embedding(ids, table).shape == (0, 8)
    out = torch.ones(5, 8, device="cuda")
    ops.embedding_grad(ids, torch.empty(0, 8, device="cuda"), out, accumulate=True)
    assert bool((out == 1).all())
    ops.embedding_grad(ids, torch.empty(0, 8, device="cuda"), out)
    assert not out.any()


@pytest.mark.parametrize("src", ["float32", "bfloat16"])
@pytest.mark.parametrize("dst", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape,dim,vocab", [((1,), 1, 1), ((7,), 33, 5), ((2, 64), 64, 1000),
                                             ((3, 5, 17), 520, 300)])
def test_lookup(src, dst, shape, dim, vocab):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(dim)
    table = torch.randn(vocab, dim, generator=gen, device="cuda").to(getattr(torch, src))
    ids = torch.randint(0, vocab, shape, generator=gen, device="cuda")
    for dtype, scale in ((torch.int64, 1.0), (torch.int32, math.sqrt(dim))):
        got = ops.embedding(ids.to(dtype), table, scale=scale, out_dtype=getattr(torch, dst))
        s = torch.tensor(scale, dtype=torch.float32)
        assert torch.equal(got, (table[ids].float() * s.cuda()).to(getattr(torch, dst)))


def test_strides():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(8)
    ids = torch.randint(0, 40, (200,), generator=gen, device="cuda")
    big = torch.randn(40, 99, generator=gen, device="cuda")
    out = torch.full((200, 77), 7.0, device="cuda")
    ops.embedding(ids, big[:, 3:67], out=out[:, 5:69])
    assert torch.equal(out[:, 5:69], big[ids, 3:67])
    assert bool((out[:, :5] == 7).all()) and bool((out[:, 69:] == 7).all())
    rows = torch.randn(200, 90, generator=gen, device="cuda")
    table = torch.full((40, 83), 7.0, device="cuda")
    ops.embedding_grad(ids, rows[:, 1:65], table[:, 9:73])
    _check_grad(torch, ids, rows[:, 1:65], table[:, 9:73], 40, 1.0)
    assert bool((table[:, :9] == 7).all()) and bool((table[:, 73:] == 7).all())
    # one row for every token
    ops.embedding_grad(ids, rows[:1, :64].contiguous().expand(200, 64).contiguous(),
                       table[:, 9:73])


def test_gradient_is_the_lookups():
    """<dout, embedding(table)> is linear in the table: its gradient times a direction is
    its value there."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(11)
    ids = _ids(torch, "text", 700, 90, gen, torch.int64)
    dout = torch.randn(700, 48, generator=gen, device="cuda")
    way = torch.randn(90, 48, generator=gen, device="cuda")
    grad = torch.empty(90, 48, device="cuda")
    ops.embedding_grad(ids, dout, grad, scale=3.0)
    value = float((ops.embedding(ids, way, scale=3.0).double() * dout).sum())
    size = float((ops.embedding(ids, way, scale=3.0).double() * dout).abs().sum())
    assert abs(float((grad.double() * way).sum()) - value) <= 1e-5 * size


def test_same_bits_twice_and_in_a_graph():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(3)
    ids = _ids(torch, "text", 3000, 500, gen, torch.int64)
    rows = torch.randn(3000, 64, generator=gen, device="cuda")
    out = torch.zeros(500, 64, device="cuda")
    ops.embedding_grad(ids, rows, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        looked = ops.embedding(ids, out)
        ops.embedding_grad(ids, rows, out)
    for k in range(3):
        ids.copy_(_ids(torch, "text", 3000, 500, gen, torch.int64))
        before = out.clone()
        graph.replay()
        torch.cuda.synchronize()
        first, rows_then = out.clone(), looked.clone()
        assert torch.equal(rows_then, before[ids])
        ops.embedding_grad(ids, rows, out)
        torch.cuda.synchronize()
        assert torch.equal(first, out), k


def test_refusals():
    torch = torch_cuda()
    from paper_1904_00962_amd import _lib, ops
    table = torch.zeros(9, 16, device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    rows = torch.zeros(4, 16, device="cuda")
    for call in (lambda: ops.embedding(ids.float(), table),
                 lambda: ops.embedding(ids, table.half()),
                 lambda: ops.embedding(ids, table, out_dtype=torch.float16),
                 lambda: ops.embedding_grad(ids, rows.half(), table)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ops.embedding(ids.cpu(), table), lambda: ops.embedding(ids, table[0]),
                 lambda: ops.embedding(ids, table.t()),
                 lambda: ops.embedding(ids, table, out=rows[:3]),
                 lambda: ops.embedding_grad(ids, rows[:2], table),
                 lambda: ops.embedding_grad(ids, rows[:, :8], table)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ops.embedding(ids, table, scale=math.inf),
                 lambda: ops.embedding_grad(ids, rows, table, scale=math.nan)):
        with pytest.raises(_lib.LambError) as e:
            call()
        assert e.value.status == _lib.LAMB_EINVAL
    with pytest.raises(_lib.LambError) as e:
        ops.embedding(ids, table, out=table[:4])
    assert e.value.status == _lib.LAMB_EOVERLAP


def test_lookup_past_one_axis_of_workgroups():
    """2^32 units of eight columns and more."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    tokens, dim, vocab = (1 << 19) + 3, 1 << 16, 5
    gen = torch.Generator(device="cuda").manual_seed(0)
    table = torch.randn(vocab, dim, generator=gen, device="cuda").to(torch.bfloat16)
    ids = torch.arange(tokens, device="cuda") % vocab
    out = ops.embedding(ids, table)
    assert out.dtype == torch.bfloat16
    for first in range(0, tokens, 1 << 16):
        part = out[first:first + (1 << 16)]
        assert torch.equal(part, table[ids[first:first + (1 << 16)]])
