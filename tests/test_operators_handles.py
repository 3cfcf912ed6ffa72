"""The handles of the operators around the step: what they keep between calls (no GPU: nothing is launched)."""
import ctypes
import gc
import sys
import threading
import weakref
from types import SimpleNamespace

import numpy
import pytest
import torch

from paper_2505_00347_amd import solo


def interleaved(calls, times=100_000):
    """Each of `calls` by a thread of its own, many times, with the threads taking turns as often as they can."""
    wrong, interval = [], sys.getswitchinterval()

    def loop(call):
        for _ in range(times):
            if not call():
                wrong.append(call)

    threads = [threading.Thread(target=loop, args=(c,)) for c in calls]
    sys.setswitchinterval(1e-6)
    try:
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(interval)
    return len(wrong)


def test_threads_that_share_an_embedding_get_the_struct_of_their_own_tensors():
    """The struct says how many rows a kernel writes: another thread's one would take it behind the end of the rows."""
    embed = solo.SoloEmbedding(10, 8, 5000, device="cpu")
    table = torch.zeros(10, 8)

    def call(n):
        rows, ids = torch.zeros(n, 8), torch.zeros(n, dtype=torch.int64)
        return lambda: embed._shape(table, rows, ids, 0).tokens == n

    assert interleaved([call(3), call(5000)]) == 0


def test_threads_that_share_log_probabilities_get_the_struct_of_their_own_tensors():
    plan = solo.SoloLogprob(5000, 8, device="cpu")

    def call(n):
        x, t = torch.zeros(n, 8), torch.zeros(n, dtype=torch.int64)
        return lambda: plan._shape(x, t).rows == n

    assert interleaved([call(3), call(5000)]) == 0


class Memory:
    """Tensors and references to the memory behind them that do not keep it."""

    def __init__(self):
        self.alive = []

    def tensor(self, n=100):
        array = numpy.zeros(n, dtype=numpy.float32)
        self.alive.append(weakref.ref(array))
        return torch.from_numpy(array)

    def count(self):
        gc.collect()
        return sum(r() is not None for r in self.alive)


@pytest.mark.parametrize("clips", [False, True])
def test_the_norms_table_keeps_the_memory_that_it_points_to(clips):
    memory = Memory()
    grads = [memory.tensor() for _ in range(3)]
    clipped = [memory.tensor() for _ in range(3)] if clips else None
    plan = solo.SoloGradNorm(grads, clipped, device="cpu")
    grads[0].data = torch.zeros(100)                       # (another memory of the same tensor)
    grads.clear()
    if clips:
        clipped[:] = [torch.zeros(100)] * 3
    assert memory.count() == (6 if clips else 3)
    del plan
    assert memory.count() == 0


def test_the_steps_table_keeps_the_memory_that_it_points_to():
    memory, cfg = Memory(), solo.make_config(4, 4, 128)
    items = [[memory.tensor(256), memory.tensor(256), solo.SoloState(256, cfg, device="cpu", init=False)] for _ in range(2)]
    for item in items:
        for name in ("m_scale", "v_scale", "v_base"):
            setattr(item[2], name, memory.tensor(2))
    table = solo.SoloMultiTable(items, cfg, device="cpu")
    items[0][1].data = torch.zeros(256)
    items[1].clear()
    items.clear()
    del item
    assert memory.count() == 10
    del table
    assert memory.count() == 0


class Streams:
    """As much of torch as a handle needs to see which stream its buffers are used on; nothing is launched."""

    def __init__(self):
        outer = self

        class Stream:
            def __init__(self, number):
                self.cuda_stream, self.waits, self.capturing = number, [], False

            def record_event(self):
                return "event of %d" % self.cuda_stream

            def wait_event(self, event):
                self.waits.append(event)

            def __enter__(self):
                self.before, outer.current = outer.current, self

            def __exit__(self, *_):
                outer.current = self.before

        self.Stream, self.current, self.external, self.device = Stream, Stream(7), [], torch.device
        self.cuda = SimpleNamespace(Stream=Stream, stream=lambda s: s, current_stream=lambda device=None: self.current, ExternalStream=self.bare,
                                    is_current_stream_capturing=lambda: self.current.capturing)

    def bare(self, number):
        self.external.append(self.Stream(number))
        return self.external[-1]

    def buffer(self):
        users = []
        return SimpleNamespace(users=users, record_stream=users.append)


@pytest.fixture
def streams(monkeypatch):
    solo.lib()
    fake = Streams()
    monkeypatch.setattr(solo, "_torch", fake)
    monkeypatch.setattr(solo, "_device_now", lambda: 0)
    monkeypatch.setattr(solo, "_stream_now", lambda device: fake.current.cuda_stream)
    return fake


def held(streams):
    handle, buffers = solo._Handle("cuda:0"), [streams.buffer(), streams.buffer()]
    handle._hold(buffers[0], None, buffers[1])
    return handle, buffers


def test_calls_on_the_stream_that_made_the_buffers(streams):
    handle, buffers = held(streams)
    assert handle._on_stream(None) == handle._on_stream(7) == handle._on_stream(streams.current) == 7
    assert not streams.current.waits and not streams.external and not any(b.users for b in buffers)


@pytest.mark.parametrize("current", [False, True])
def test_the_first_call_on_another_stream_waits_for_the_buffers(streams, current):
    """Their memory may be a block that work enqueued before still uses; and the allocator must not give it away under this stream's work."""
    handle, buffers = held(streams)
    side = streams.Stream(8)
    if current:
        streams.current = side
    for _ in range(2):
        assert handle._on_stream(None if current else side) == 8
        assert side.waits == ["event of 7"] and all(b.users == [side] for b in buffers)
    handle._hold(buffers[0])                               # (made anew)
    assert handle._on_stream(side) == 8
    assert side.waits == (["event of 7"] if current else ["event of 7"] * 2)


@pytest.mark.parametrize("stream", [9, SimpleNamespace(cuda_stream=9)])
def test_a_stream_that_is_not_torchs_is_not_remembered(streams, stream):
    """It may be destroyed before the buffers are, and its number be another's."""
    handle, buffers = held(streams)
    for k in (1, 2):
        assert handle._on_stream(stream) == 9
        assert len(streams.external) == k and streams.external[-1].cuda_stream == 9 and streams.external[-1].waits == ["event of 7"]
    assert not any(b.users for b in buffers)
    for none in (SimpleNamespace(cuda_stream=None), SimpleNamespace(cuda_stream=ctypes.c_void_p(0)), 0):
        assert handle._on_stream(none) == 0


def test_a_captured_call_waits_for_nothing_outside_of_the_graph(streams):
    handle, buffers = held(streams)
    side = streams.Stream(8)
    side.capturing = True
    assert handle._on_stream(side) == 8
    assert not side.waits and not any(b.users for b in buffers)
    side.capturing = False
    assert handle._on_stream(side) == 8
    assert side.waits == ["event of 7"] and all(b.users == [side] for b in buffers)


def test_a_handle_without_buffers_takes_any_stream(streams):
    handle = solo._Handle("cuda:0")
    assert handle._on_stream(None) == 7 and handle._on_stream(9) == 9 and handle._on_stream(streams.Stream(8)) == 8


def test_a_handle_runs_on_its_own_device(streams, monkeypatch):
    handle, _ = held(streams)
    monkeypatch.setattr(solo, "_device_now", lambda: 1)
    for stream in (None, 7, streams.current):
        with pytest.raises(ValueError, match="cuda:0"):
            handle._on_stream(stream)
    monkeypatch.setattr(solo, "_device_now", lambda: 0)
    other = streams.Stream(7)
    other.device_index = 1
    with pytest.raises(ValueError, match="stream on cuda:0"):
        handle._on_stream(other)
    other.device_index = 0
    assert handle._on_stream(other) == 7


def on(device, tensor):
    class There(torch.Tensor):
        pass

    There.device = property(lambda self: torch.device(device))
    return tensor.as_subclass(There)


def test_tensors_of_another_device_are_refused():
    """Of another GPU, too: the call runs on the handle's."""
    embed = solo.SoloEmbedding(10, 8, 4, device="cuda:0")
    table, ids, rows = torch.zeros(10, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4, 8)
    here = [on("cuda:0", t) for t in (table, rows, ids)]
    assert embed._shape(*here, 0).tokens == 4
    for k, t in enumerate((table, rows, ids)):
        for other in (t, on("cuda:1", t)):
            with pytest.raises(ValueError, match="cuda:0"):
                embed._shape(*here[:k], other, *here[k + 1:], 0)
    with pytest.raises(ValueError, match="cuda:0"):
        solo._row_weights(on("cuda:1", torch.zeros(4)), 4, "grad_logprob", torch.device("cuda:0"))


def test_a_handle_on_the_host_runs_nothing():
    """Host addresses are nothing for a kernel: every call is refused, also one that fits."""
    table, ids, rows = torch.zeros(10, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4, 8)
    embed, plan = solo.SoloEmbedding(10, 8, 4, device="cpu"), solo.SoloLogprob(4, 8, device="cpu")
    norm, w = solo.SoloGradNorm([table], [table.clone()], device="cpu"), torch.zeros(4)
    for call in (lambda: embed.lookup(table, ids, rows, stream=0), lambda: embed.grad(rows, ids, table, stream=0),
                 lambda: plan.forward(rows, ids, stream=0), lambda: plan.grad(rows, ids, w, None, rows, stream=0),
                 lambda: plan.forward_grad(rows, ids, w, None, rows, stream=0), lambda: norm.norm(stream=0), lambda: norm.clip(1.0, stream=0)):
        with pytest.raises(ValueError):
            call()


def test_a_gradient_needs_the_sums_of_its_rows(monkeypatch):
    """grad() reads entropy and stats of forward(): of as many rows, with the same scale, and never of forward_grad()."""
    calls = []
    monkeypatch.setattr(solo, "_operation", lambda name, check, *args: calls.append((name, args)))
    plan, w = solo.SoloLogprob(4, 8, device="cpu"), torch.zeros(4)
    monkeypatch.setattr(plan, "_on_stream", lambda stream: 0)
    x, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)

    def refused(n):
        with pytest.raises(ValueError, match="forward"):
            plan.grad(x[:n], t[:n], w[:n], None, x[:n])

    refused(1)
    plan.forward_grad(x, t, w, None, x)
    refused(1)
    plan.forward(x[:3], t[:3])
    refused(4)
    plan.grad(x[:3], t[:3], w[:3], None, x[:3])
    plan.scale = 2.0
    refused(3)
    plan.forward(x, t)
    plan.forward_grad(x[:2], t[:2], w[:2], None, x[:2])
    plan.grad(x, t, w, None, x)
    assert [name for name, _ in calls] == ["solo_logprob_with_grad", "solo_logprob", "solo_logprob_grad", "solo_logprob", "solo_logprob_with_grad", "solo_logprob_grad"]
    for name, args in calls:
        read = args[2:4] if name == "solo_logprob_grad" else (args[3], args[7]) if name == "solo_logprob" else ()
        assert all(a is b for a, b in zip(read, (plan.entropy, plan.stats)))
        assert name != "solo_logprob_with_grad" or not any(a is b for a in args for b in (plan.entropy, plan.stats))
