"""The operators around the step at sizes behind the lines of their dispatch, against plain implementations in 64 bits."""
import pytest
import torch

from paper_2505_00347_amd import solo

pytestmark = pytest.mark.gpu


def test_as_many_tokens_as_a_gradient_takes():
    """The parts of frequent tokens are more than one launch has workgroups for.  Whole numbers, whose sums are exact."""
    n, vocab = (1 << 28) - 1, 70_000
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, vocab, (n,), generator=gen, device="cuda", dtype=torch.int32)
    rows = torch.randint(-8, 9, (n, 1), generator=gen, device="cuda", dtype=torch.int8).bfloat16()
    out = solo.SoloEmbedding(vocab, 1, n).grad(rows, ids, torch.empty((vocab, 1), device="cuda"))
    want = torch.zeros(vocab, dtype=torch.float64, device="cuda")
    for at in range(0, n, 1 << 26):
        want.index_add_(0, ids[at:at + (1 << 26)], rows[at:at + (1 << 26), 0].double())
    assert torch.equal(out[:, 0].double(), want)
