"""The handles of the operators around the step: what they keep between calls (no GPU: nothing is launched)."""
import gc
import sys
import threading
import weakref

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
