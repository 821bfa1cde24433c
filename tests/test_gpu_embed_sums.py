"""The sum of an id that very many tokens share.

Tolerance. Tokens are summed 16 at a time, 64 of these sums at a time, and then these: an
element is in at most 16 + 64 + tokens / 1024 + 2 additions, each off by 2^-24 of its
result at most, and a bf16 result by 2^-8. Rows are the same for every token, so that
roundings do not cancel."""

import math

import pytest

from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("table", ["float32", "bfloat16"])
@pytest.mark.parametrize("tokens", [1000, 1040, 40001, 1 << 20])
def test_like_rows_of_one_id(table, tokens):
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    row = torch.linspace(0.1, 7.3, 72, device="cuda")
    ids = torch.full((tokens,), 5, device="cuda")
    ids[::1001] = 6
    kept = int((ids == 5).sum())
    rows = row.repeat(tokens, 1)
    for old in (0.0, 3.0):
        out = torch.full((9, 72), old or math.nan, dtype=getattr(torch, table), device="cuda")
        ops.embedding_grad(ids, rows, out, accumulate=old != 0.0)
        off = (out[5].double() / (row.double() * kept + old) - 1).abs()
        bound = (16 + 64 + tokens / 1024 + 2) * 2.0 ** -24
        assert float(off.max()) <= bound + (2.0 ** -8 if table == "bfloat16" else 0.0)
