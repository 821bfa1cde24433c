"""The example model trains: from the loss of a uniform guess down, with every operator
and both optimizers in the loop, and the same losses from the same seed."""

import importlib.util
import math
import os

import pytest

from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "tied_lm.py")


def test_the_example_learns():
    torch_cuda()
    spec = importlib.util.spec_from_file_location("tied_lm", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.train(steps=60, vocab=500, dim=64, tokens=1024)
    assert abs(losses[0] - math.log(500)) < 0.5
    assert all(math.isfinite(v) for v in losses)
    assert sum(losses[-5:]) / 5 < 0.75 * losses[0], losses[::10]
