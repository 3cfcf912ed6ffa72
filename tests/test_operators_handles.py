"""The handles of the operators around the step: what they keep between calls (no GPU: nothing is launched)."""
import sys
import threading

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
