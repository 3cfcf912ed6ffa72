"""Layer norm, distillation and sampling as they are used together: between the embedding and the step, behind a teacher, token by token."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

# What rounds to bfloat16 on the way (half a step, 2^-8, each): the scaled rows, the norm's output, the logits (of magnitude up to 20, in the gradient's
# exponent: 0.04 each, of random sign), their gradient, the products' results.  Relative to a whole gradient's norm the independent
# roundings of its entries average: far below 0.05.
NEAR = 0.05


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def exact_gradients(model, ids, slope):
    """Gradients of embedding, head, weight and bias for the logits' gradient slope(logits), in 64 bits."""
    embedding, head, weight, bias = (w.double().requires_grad_() for w in model.weights)
    rows = embedding[ids] * math.sqrt(model.dim)
    centred = rows - rows.mean(1, keepdim=True)
    hidden = centred / (centred.square().mean(1, keepdim=True) + 1e-5).sqrt() * weight + bias
    logits = hidden @ head.t()
    logits.backward(slope(logits.detach()))
    return [t.grad for t in (embedding, head, weight, bias)], logits.detach()


def model_of(**more):
    from paper_2505_00347_amd import bigram
    return bigram.Bigram(**{**dict(vocab=600, dim=96, tokens=512, norm=True), **more})


def test_gradients_through_the_norm():
    from paper_2505_00347_amd import bigram
    model = model_of()
    for w in model.weights[2:]:
        w.add_(0.3 * torch.randn(96, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)))
    ids, targets = bigram.text(600, 512, 1)

    def slope(logits):
        p = torch.softmax(logits, 1)
        p[torch.arange(512), targets] -= 1.0
        return p / 512
    want, logits = exact_gradients(model, ids, slope)
    logprob, norm = model.step(ids, targets)
    assert float((logprob.double() - torch.log_softmax(logits, 1)[torch.arange(512), targets]).abs().mean()) < 0.05
    for got, exact in zip(model.grads, want):
        assert off(got, exact) < NEAR
    assert abs(norm.item() / math.sqrt(sum(float(g.double().square().sum()) for g in model.grads)) - 1) < 1e-6
    assert all(bool(torch.isfinite(p).all()) for p in model.params)


def test_a_student_follows_its_teachers_alternatives():
    from paper_2505_00347_amd import bigram
    teacher, student = model_of(dim=128, norm=False, seed=2), model_of(seed=3)
    ids, _ = bigram.text(600, 512, 1)
    value, token = (t.clone() for t in teacher.alternatives(ids, 20))

    def slope(logits):
        q, p = torch.softmax(logits, 1), value.double().exp()
        among = torch.zeros_like(q).scatter_(1, token.long(), 1.0) > 0
        left = 1 - p.sum(1, keepdim=True)
        tail = torch.where(among, 0.0, q)
        target = torch.zeros_like(q).scatter_(1, token.long(), p) + tail / tail.sum(1, keepdim=True) * left
        return (q - target) / 512
    want, logits = exact_gradients(student, ids, slope)
    loss, norm = student.learn(ids, value, token)
    assert bool((loss > -1e-3).all()) and bool(torch.isfinite(loss).all())
    for got, exact in zip(student.grads, want):
        assert off(got, exact) < NEAR


def test_a_text_is_drawn_token_by_token():
    model = model_of(tokens=64)
    ids = torch.arange(20, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    uniform = torch.rand((6, 20), generator=gen, device="cuda")
    tokens, logprobs = model.write(ids, uniform, temperature=0.8, top_k=50, top_p=0.9)
    assert tokens.shape == (6, 20) and bool(((tokens >= 0) & (tokens < 600)).all()) and bool((logprobs <= 0).all())
    again = model.write(ids, uniform, temperature=0.8, top_k=50, top_p=0.9)
    assert torch.equal(again[0], tokens) and torch.equal(again[1], logprobs)
    greedy, _ = model.write(ids, uniform, temperature=0.0)
    now = ids
    for step in greedy:                                    # each is the largest logit's column, as the alternatives have it
        assert torch.equal(step, model.alternatives(now, 1)[1][:, 0].long())
        now = step


def test_the_example_runs(capsys):
    from paper_2505_00347_amd import bigram
    bigram.main(steps=4)
    out = capsys.readouterr().out
    assert "a text behind 100" in out and "student, step   1" in out


def test_two_runs_are_the_same():
    from paper_2505_00347_amd import bigram
    results = []
    for _ in range(2):
        teacher, student = model_of(norm=False, seed=2), model_of(seed=3)
        for k in range(1, 4):
            ids, targets = bigram.text(600, 512, k)
            teacher.step(ids, targets)
            loss, norm = student.learn(ids, *teacher.alternatives(ids, 8))
        results.append((loss.clone(), norm.clone(), *student.params, *teacher.params))
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_a_decoding_step_in_a_graph():
    """Lookup, norm, product and sampling captured together: the token feeds the next replay."""
    from paper_2505_00347_amd import solo
    model = model_of(tokens=8)
    start, uniform = torch.arange(8, device="cuda"), torch.rand((5, 8), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    ids, u = start.clone(), uniform[0].clone()
    sampler = solo.SoloSampler(8, 600, top_p=0.95)

    def decode():
        ids.copy_(sampler.sample(model._forward(ids), u)[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        decode()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decode()
    ids.copy_(start)
    replayed = []
    for k in range(5):
        u.copy_(uniform[k])
        graph.replay()
        replayed.append(ids.clone())
        torch.cuda.synchronize()
    assert torch.equal(torch.stack(replayed), model.write(start, uniform, top_p=0.95)[0])
