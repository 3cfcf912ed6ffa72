"""The operators around the step and the step itself, as one training program."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_training_learns_the_chain():
    """The first loss is that of a random model, the gradient is the loss's, and 120 steps find most of what there is to learn."""
    from paper_2505_00347_amd import bigram
    model = bigram.Bigram()
    ids, targets = bigram.text(model.vocab, model.tokens, 1)
    rows = model.weights[0].double()[ids] * 16.0
    logits = rows @ model.weights[1].double().t()
    want = -torch.log_softmax(logits, 1)[torch.arange(model.tokens), targets].mean()
    p = torch.softmax(logits, 1)
    p[torch.arange(model.tokens), targets] -= 1.0
    grad_head = p.t() @ rows / model.tokens
    grad_rows = p @ model.weights[1].double() / model.tokens * 16.0
    grad_embedding = torch.zeros_like(grad_head).index_add_(0, ids, grad_rows)
    logprob, norm = model.step(ids, targets)
    # bf16 logits (8 bits) of magnitude up to 60: 0.1 each, averaged; bf16 gradients
    assert abs(-logprob.double().mean() - want) < 0.02
    for got, exact in zip(model.grads, (grad_embedding, grad_head)):
        assert float((got.double() - exact).norm() / exact.norm()) < 0.05
    assert abs(norm.item() / math.sqrt(sum(float(g.double().square().sum()) for g in model.grads)) - 1) < 1e-6
    for k in range(2, 121):
        logprob, _ = model.step(*bigram.text(model.vocab, model.tokens, k))
    best = 0.2 * math.log(5 * model.vocab) + 0.8 * math.log(1 / 0.8)
    assert best - 0.1 < -logprob.mean().item() < 0.5 * want.item()
    ids = torch.arange(100, device="cuda")
    value, token = model.successors(ids, top=2)
    assert float((token[:, 0] == bigram.follows(ids, model.vocab)).float().mean()) > 0.9
    assert bool((value[:, 0] >= value[:, 1]).all())


def test_two_runs_are_the_same():
    from paper_2505_00347_amd import bigram
    results = []
    for _ in range(2):
        model = bigram.Bigram(vocab=500, dim=64, tokens=1024)
        for k in range(1, 6):
            logprob, norm = model.step(*bigram.text(model.vocab, model.tokens, k))
        results.append((logprob.clone(), norm.clone(), *model.params, *model.weights))
    assert all(torch.equal(a, b) for a, b in zip(*results))
