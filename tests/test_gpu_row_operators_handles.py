"""Handles of layer norm, distillation and sampling on streams of their own.  What is checked is order, on the host: the current stream is kept busy by a kernel that
touches no memory."""
import time

import pytest
import torch

from paper_2505_00347_amd import solo
from test_gpu_operators_handles import ticks

pytestmark = pytest.mark.gpu


def layer_of(x, t, stream):
    plan, out = solo.SoloLayerNorm(*x.shape), [torch.empty_like(x), torch.empty_like(x), torch.empty(x.shape[1], device="cuda"), torch.empty(x.shape[1], device="cuda")]

    def run(stream=None):
        plan.forward(x, None, None, out[0], stream=stream)
        plan.grad(x, x, None, *out[1:], stream=stream)
        return out
    return run, run(stream)


def distill_of(x, t, stream):
    # (what is made here on the current stream comes before the handle: its event says when the buffers are ready, and with them all that was enqueued before)
    value, weight = x[:, :3].log_softmax(1) - 0.1, torch.ones(len(x), device="cuda")
    token = torch.stack([t, (t + 1) % x.shape[1], (t + 2) % x.shape[1]], 1)
    plan, out = solo.SoloDistill(*x.shape, 3, rest=True), torch.empty_like(x)

    def run(stream=None):
        loss = plan.forward(x, value, token, stream=stream)
        return loss, plan.grad(x, value, token, weight, out, stream=stream)
    return run, run(stream)


def sample_of(x, t, stream):
    uniform = (t.float() + 0.5) / x.shape[1]
    plan = solo.SoloSampler(*x.shape, top_p=0.9)
    run = lambda stream=None: plan.sample(x, uniform, stream=stream)       # noqa: E731
    return run, run(stream)


@pytest.mark.parametrize("way", ["argument", "number", "current"])
@pytest.mark.parametrize("call", [layer_of, distill_of, sample_of])
def test_the_first_call_comes_behind_the_work_that_its_buffers_memory_may_still_have(call, way):
    x, t = torch.randn((600, 64), device="cuda"), torch.randint(0, 64, (600,), device="cuda")
    want = [v.clone() for v in call(x, t, None)[1]]
    side = torch.cuda.Stream()
    ticks()
    torch.cuda.synchronize()
    torch.cuda._sleep(ticks())
    busy = torch.cuda.Event()
    busy.record()
    if way != "current":
        _, got = call(x, t, side if way == "argument" else side.cuda_stream)
    else:                                                  # the buffers are made on the one, the call comes on the other
        with pytest.MonkeyPatch.context() as patch:
            patch.setattr(solo, "_operation", lambda *args: None)
            run, _ = call(x, t, None)
        with torch.cuda.stream(side):
            got = run()
    done = torch.cuda.Event()
    done.record(side)
    time.sleep(0.01)
    assert busy.query() or not done.query()
    side.synchronize()
    assert busy.query()
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want))


def test_forward_and_gradient_in_one_call_leaves_what_grad_takes():
    x, other = torch.randn((40, 300), device="cuda"), torch.randn((40, 300), device="cuda") * 5
    value, token, a = torch.randn((40, 6), device="cuda"), torch.randint(0, 300, (40, 6), device="cuda"), torch.rand(40, device="cuda")
    plan = solo.SoloDistill(40, 300, 6)
    plan.forward(x, value, token)
    want = plan.grad(x, value, token, a, torch.empty_like(x)).clone()
    plan.forward(x, value, token)
    plan.forward_grad(other, value, token, a, torch.empty_like(x))
    assert torch.equal(plan.grad(x, value, token, a, torch.empty_like(x)), want)


def test_two_graphs_of_one_handle_replayed_one_after_the_other():
    """They share the handle's buffers and, of layer norm, the workspace."""
    x, dy = torch.randn((2000, 500), device="cuda"), torch.randn((2000, 500), device="cuda")
    w = torch.randn(500, device="cuda")
    plan, out = solo.SoloLayerNorm(2000, 500), [[torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)] for _ in range(3)]

    def run(x, dy, out):
        plan.forward(x, w, None, out[0])
        plan.grad(dy, x, w, *out[1:])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(x, dy, out[0])
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for k, rows in ((0, 2000), (1, 700)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            run(x[:rows], dy[:rows], [t[:rows] if t.dim() == 2 else t for t in out[k]])
    for n in range(3):
        x.copy_(torch.randn((2000, 500), device="cuda"))
        for k, rows in ((n % 2, (2000, 700)[n % 2]), (1 - n % 2, (2000, 700)[1 - n % 2])):
            graphs[k].replay()
        torch.cuda.synchronize()
        got = [[t.clone() for t in o] for o in out[:2]]
        for k, rows in ((0, 2000), (1, 700)):
            run(x[:rows], dy[:rows], [t[:rows] if t.dim() == 2 else t for t in out[2]])
            assert all(torch.equal(a[:rows] if a.dim() == 2 else a, b[:rows] if b.dim() == 2 else b) for a, b in zip(got[k], out[2]))
