"""Handles of the operators around the step on streams of their own.  What is checked is order, on the host: the current stream is kept busy
by a kernel that touches no memory."""
import functools
import time

import pytest
import torch

from paper_2505_00347_amd import solo

pytestmark = pytest.mark.gpu


@functools.lru_cache(None)
def ticks():
    """Of a kernel that only waits, for 0.1 seconds."""
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    for _ in range(2):
        begin.record()
        torch.cuda._sleep(1_000_000)
        end.record()
        torch.cuda.synchronize()
    return int(1_000_000 * 100 / begin.elapsed_time(end))


def logprob_of(x, t, stream):
    plan = solo.SoloLogprob(*x.shape, top=3, rank=True)
    return plan, plan.forward(x, t, stream=stream)


def gradient_of(dy, ids, stream):
    plan = solo.SoloEmbedding(70, dy.shape[1], len(ids))
    return plan, (plan.grad(dy, ids, torch.empty((70, dy.shape[1]), device="cuda"), stream=stream),)


def norm_of(x, t, stream):
    plan = solo.SoloGradNorm([x], [torch.empty_like(x)])
    return plan, (*plan.clip(1.0, stream=stream), plan._keep[1])


@pytest.mark.parametrize("way", ["argument", "number", "current"])
@pytest.mark.parametrize("call", [logprob_of, gradient_of, norm_of])
def test_the_first_call_comes_behind_the_work_that_its_buffers_memory_may_still_have(call, way):
    """A stream's first call waits for the stream that made the buffers, and leaves them to no one else before it is done."""
    x, t = torch.randn((600, 64), device="cuda"), torch.randint(0, 64, (600,), device="cuda")
    want = [v.clone() for v in call(x, t, None)[1]]
    side = torch.cuda.Stream()
    ticks()
    torch.cuda.synchronize()
    torch.cuda._sleep(ticks())
    busy = torch.cuda.Event()
    busy.record()
    if way != "current":
        plan, got = call(x, t, side if way == "argument" else side.cuda_stream)
    else:                                                  # the buffers are made on the one, the call comes on the other
        real = solo._operation
        with pytest.MonkeyPatch.context() as patch:
            patch.setattr(solo, "_operation", lambda *args: None)
            plan, got = call(x, t, None)
        with torch.cuda.stream(side):
            if call is logprob_of:
                got = plan.forward(x, t)
            elif call is gradient_of:
                plan.grad(x, t, got[0])
            else:
                plan.clip(1.0)
        assert solo._operation is real
    done = torch.cuda.Event()
    done.record(side)
    time.sleep(0.01)
    # (the norm's table is copied from the host, which by itself waits for the current stream)
    assert call is norm_of or not busy.query()
    assert busy.query() or not done.query()
    side.synchronize()
    assert busy.query()
    assert all(torch.equal(g, w) for g, w in zip(got, want))


def test_buffers_under_work_of_another_stream_are_not_given_away():
    dy, ids = torch.randn((600, 64), device="cuda"), torch.randint(0, 70, (600,), device="cuda")
    out, side = torch.empty((70, 64), device="cuda"), torch.cuda.Stream()
    plan = solo.SoloEmbedding(70, 64, 600)
    plan.grad(dy, ids, out)
    ticks()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(ticks())
    plan.grad(dy, ids, out, stream=side)
    place, size = plan.workspace.data_ptr(), plan.workspace.numel()
    del plan
    other = torch.empty(size, dtype=torch.uint8, device="cuda")
    assert other.data_ptr() != place
    side.synchronize()


def test_both_gradient_calls_on_one_handle():
    """forward_grad() on other rows between forward() and grad() does not change what grad() gives."""
    x, other = torch.randn((40, 300), device="cuda"), torch.randn((40, 300), device="cuda") * 5
    t, a = torch.randint(0, 300, (40,), device="cuda"), torch.rand(40, device="cuda")
    plan = solo.SoloLogprob(40, 300)
    plan.forward(x, t)
    want = plan.grad(x, t, a, a, torch.empty_like(x)).clone()
    plan.forward(x, t)
    _, entropy, _ = plan.forward_grad(other, t, a, a, torch.empty_like(x))
    assert torch.equal(plan.grad(x, t, a, a, torch.empty_like(x)), want)
    assert not torch.equal(entropy, plan.entropy)
