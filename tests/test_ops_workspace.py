"""The cross entropy's workspace against the bytes that the header states, over the sizes
that it accepts (host code, no GPU)."""

import pytest

from paper_1904_00962_amd import _ops, build

A = 1 << 40
MIB = 1 << 20
SIZES = [1, 7, 8, 64, 1000, 8192, 32768, 32769, 50257, 131072, 200000, 300000, 327680, 327681,
         1 << 20, 3000001, 1 << 24]


@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("dim", [1, 64, 250, 1024, 1600, 65536])
def test_workspaces_are_within_the_stated_bytes(dim, aligned):
    if build.is_stale():
        build.build()
    d = (dim + 7) // 8 * 8
    copied = not aligned or dim % 8
    stride = dim if aligned else dim + 1
    for tokens in SIZES:
        for vocab in SIZES:
            x = _ops.lamb_xent(A, A + (1 << 44), A + (1 << 45), stride, stride, tokens, vocab,
                               dim, -100, _ops.LAMB_DTYPE_I64, 0)
            both = (2 * d + 8) * tokens + (2 * d * vocab if copied else 0) + 4096
            forward = both + 8 * tokens * -(-vocab // 64) + 4 * tokens
            backward = both + max(160 * MIB, 512 * tokens) + 4 * d * tokens + 128 * MIB + (
                10240 * d if tokens > 32768 else 0)
            assert _ops.lamb_xent_workspace(x, False) <= forward, (tokens, vocab)
            assert _ops.lamb_xent_workspace(x, True) <= backward, (tokens, vocab)


def test_a_large_call_takes_large_tiles():
    x = _ops.lamb_xent(A, A + (1 << 44), A + (1 << 45), 1024, 1024, 1 << 20, 50257, 1024, -100,
                       _ops.LAMB_DTYPE_I64, 0)
    parts = _ops.lamb_xent_workspace(x, False) - (2 * 1024 + 12) * (1 << 20)
    assert 8 * (1 << 20) * 197 <= parts <= 1.6 * 2 ** 30
