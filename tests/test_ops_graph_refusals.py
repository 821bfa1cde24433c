"""A tensor whose gradient would be lost is refused before anything else is looked at, with
the function that gives the gradient; on the CPU."""

import re

import pytest
import torch

from paper_1904_00962_amd import ops


@pytest.mark.parametrize("name,call", [
    ("rms_norm", lambda p, t: ops.rms_norm(p)),
    ("rms_norm", lambda p, t: ops.rms_norm(t, p[0])),
    ("rms_norm", lambda p, t: ops.rms_norm(t, residual=p)),
    ("rms_norm", lambda p, t: ops.rms_norm(t, out=p)),
    ("rms_norm", lambda p, t: ops.rms_norm(t, residual=t, summed=p)),
    ("rms_norm_fp8", lambda p, t: ops.rms_norm_fp8(p)),
    ("rms_norm_fp8", lambda p, t: ops.rms_norm_fp8(t, p[0])),
    ("rms_norm_fp8", lambda p, t: ops.rms_norm_fp8(t, residual=p)),
    ("rms_norm_fp8", lambda p, t: ops.rms_norm_fp8(t, residual=t, summed=p)),
    ("rms_norm_fp8", lambda p, t: ops.rms_norm_fp8(t, scales=p)),
    ("rms_norm_fp8", lambda p, t: ops.rms_norm_fp8(t, out=p)),
    ("linear_cross_entropy", lambda p, t: ops.linear_cross_entropy(p, t, t[:, 0])),
    ("embedding", lambda p, t: ops.embedding(t[:, 0], p)),
])
def test_lost_gradients(name, call):
    tensor = torch.zeros(3, 8)
    with pytest.raises(ValueError, match="detach") as e:
        call(tensor.clone().requires_grad_(), tensor)
    said, instead = re.match(r"(\w+) records .* from (\w+)$", str(e.value)).groups()
    assert said == name and callable(getattr(ops, instead))
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
        ops.rms_norm(tensor.requires_grad_())
