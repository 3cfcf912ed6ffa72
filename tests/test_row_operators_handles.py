"""Handles whose buffers are made at different times, on different streams (no GPU: nothing is launched)."""
import pytest
import torch

from paper_2505_00347_amd import solo
from test_operators_handles import on, streams  # noqa: F401  (a fixture)


@pytest.fixture
def layer(streams, monkeypatch):  # noqa: F811
    """A layer norm's handle made on stream 7, its two calls, and the operations they ask for."""
    streams.float32, streams.bfloat16, streams.uint8 = torch.float32, torch.bfloat16, torch.uint8
    streams.empty = lambda *shape, **kind: streams.buffer()
    calls = []
    monkeypatch.setattr(solo, "_operation", lambda name, check, *args: calls.append((name, args[-1])))
    plan, x = solo.SoloLayerNorm(4, 8, device="cuda:0"), on("cuda:0", torch.zeros(4, 8))
    dw = on("cuda:0", torch.zeros(8))
    plan.calls = calls
    plan.run_forward = lambda stream=None: plan.forward(x, None, None, x, stream=stream)
    plan.run_grad = lambda stream=None: plan.grad(x, x, None, x, dw, None, stream=stream)
    return plan


def test_a_gradient_on_another_stream_than_the_handles(layer, streams):  # noqa: F811
    """The workspace is made there, the sums of forward() were made on the stream of the constructor: the allocator has to learn of both."""
    home, side = streams.current, streams.Stream(8)
    layer.run_forward()
    streams.current = side
    layer.run_grad()
    assert layer.calls == [("solo_layernorm", 7), ("solo_layernorm_grad", 8)]
    assert layer.stats.users == [side] and side.waits == ["event of 7"] and not layer.workspace.users
    layer.run_grad()                                       # (what is known is not done again)
    assert layer.stats.users == [side] and side.waits == ["event of 7"]
    streams.current = home
    layer.run_forward()
    assert layer.workspace.users == [home] and home.waits == ["event of 8"] and layer.stats.users == [side]


def test_a_third_stream_waits_for_all_buffers(layer, streams):  # noqa: F811
    side, third = streams.Stream(8), streams.Stream(9)
    layer.run_forward(third)
    assert third.waits == ["event of 7"] and layer.stats.users == [third]
    streams.current = side
    layer.run_grad()
    streams.current = third
    layer.run_grad()
    assert layer.workspace.users == [third] and "event of 8" in third.waits and side in layer.stats.users


def test_a_first_gradient_that_is_captured(layer, streams):  # noqa: F811
    """It waits for nothing outside of the graph, and the stream is not taken for the home of the sums when it runs calls of its own later."""
    home, side = streams.current, streams.Stream(8)
    layer.run_forward()
    streams.current, side.capturing = side, True
    layer.run_grad()
    assert not side.waits and not layer.stats.users
    side.capturing = False
    layer.run_grad()
    assert layer.stats.users == [side] and side.waits == ["event of 7"]
    streams.current = home
    layer.run_grad()
    assert layer.workspace.users == [home]


def test_a_workspace_made_on_the_handles_stream(layer, streams):  # noqa: F811
    layer.run_forward()
    layer.run_grad()
    assert not streams.current.waits and not layer.stats.users and not layer.workspace.users
    side = streams.Stream(8)
    layer.run_grad(side)
    assert layer.stats.users == [side] and layer.workspace.users == [side] and set(side.waits) == {"event of 7"}
