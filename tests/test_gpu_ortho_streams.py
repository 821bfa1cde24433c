"""Calls of one plan on several streams, which share its workspace: each waits for the one
before, and the results are those of one stream."""

import pytest

from gpu_harness import torch_cuda
from test_gpu_ortho import _make, _muon_state

pytestmark = pytest.mark.gpu

CYCLES = 5_000_000  # milliseconds, beside calls of about 0.1


def test_a_call_waits_for_the_one_on_another_stream():
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gs = _make(torch, [(130, 70), (70, 300), (256, 256)], torch.float32)
    want = [o.clone() for o in ops.Orthogonalizer(gs).run()]
    plan = ops.Orthogonalizer(gs)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    before, after = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    torch.cuda.synchronize()
    for first, second in ((a, b), (b, a), (a, torch.cuda.default_stream())):
        with torch.cuda.stream(first):
            torch.cuda._sleep(CYCLES)
            before.record()
            plan.run()
        with torch.cuda.stream(second):
            plan.run()
            after.record()
        torch.cuda.synchronize()
        assert before.elapsed_time(after) > 0
        assert all(torch.equal(x, y) for x, y in zip(want, plan.outputs))


def test_muon_steps_that_change_streams():
    torch = torch_cuda()
    from paper_1904_00962_amd import Muon
    shapes = [(64, 147), (200, 96), (33, 1)]
    xs, gs, ms = _muon_state(torch, shapes, torch.bfloat16)
    ys, ns = [x.clone() for x in xs], [m.clone() for m in ms]
    one = Muon(xs, gs, m=ms, lr=0.02, skip_nonfinite=True)
    for _ in range(6):
        one.step()
    two = Muon(ys, gs, m=ns, lr=0.02, skip_nonfinite=True)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for k in range(6):
        with torch.cuda.stream(streams[k % 3]):
            torch.cuda._sleep(CYCLES * (2 - k % 3) // 4)
            two.step()
    torch.cuda.synchronize()
    for p, q in zip(xs + ms, ys + ns):
        assert torch.equal(p, q)


def test_a_captured_call_between_eager_ones():
    """The graph's replays are ordered here by their stream; eager calls on another one
    follow through an event of the caller's."""
    torch = torch_cuda()
    from paper_1904_00962_amd import ops
    gs = _make(torch, [(100, 60), (128, 128)], torch.float32)
    plan = ops.Orthogonalizer(gs)
    want = [o.clone() for o in plan.run()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run()
    side = torch.cuda.Stream()
    for _ in range(3):
        for o in plan.outputs:
            o.zero_()
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            plan.run()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, plan.outputs))
