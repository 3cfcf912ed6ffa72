"""Distillation from a teacher's alternatives on the GPU against a plain implementation in 64 bits.

Bounds.  U = 2^-24, r: half a step of the logits' type.  An exponential of a difference d (in units of ln 2, up to 1.5 |d| of them) is off by
8 U (1 + |d|); a thread adds up to cols / 256 + 8 of them and at most 24 steps join the threads: a sum is off by A = 8 U (1 + reach) +
(cols / 256 + 32) U, `reach` being how far the logits that count lie below the largest."""
import math

import pytest
import torch

from paper_2505_00347_amd import solo
from test_gpu_operators import ROUND, TYPES, U, generator, randn, strided, within

pytestmark = pytest.mark.gpu
NO_REST = 2.0 ** -20


def exact(x, value, token, weight, rest, scale, teacher_scale):
    """Loss, gradient and their bounds, in 64 bits on the CPU."""
    x, value, token, a = x.double().cpu(), value.double().cpu(), token.long().cpu(), weight.double().cpu()[:, None]
    rows, cols = x.shape
    live = (token >= 0) & (token < cols) & (value > -math.inf)
    row = live.any(1)
    x = torch.where(row[:, None], x, 0.0)
    z = x * scale
    m = z.amax(1, keepdim=True)
    empty = row & (m[:, 0] == -math.inf)
    d = torch.where(empty[:, None], -math.inf, z - torch.where(empty[:, None], 0.0, m))
    e = d.exp()
    s = e.sum(1, keepdim=True)
    at = torch.where(live, token, 0)
    v = torch.where(live, value * (1.0 if rest else teacher_scale), -math.inf)
    log_p = v if rest else torch.where(row[:, None], v - torch.logsumexp(v, 1, keepdim=True), -math.inf)
    p = torch.where(live, log_p.exp(), 0.0)
    d_k = d.gather(1, at)
    terms = torch.where(p > 0, p * (log_p - d_k + s.log()), 0.0)
    loss, size = terms.sum(1), torch.where(p > 0, p * (log_p.abs() + d_k.abs() + s.log().abs()), 0.0).sum(1)
    left = (1 - p.sum(1, keepdim=True)).clamp(min=0) if rest else torch.zeros((rows, 1), dtype=torch.float64)
    left = torch.where(left < NO_REST, 0.0, left)
    among = torch.zeros((rows, cols), dtype=torch.float64).scatter_add_(1, at, live.double()) > 0
    s_rest = torch.where(among, 0.0, e).sum(1, keepdim=True)
    tail = torch.where(left > 0, left * (left.log() - (s_rest / s).log()), 0.0)[:, 0]
    loss = torch.where(row, torch.where(empty, math.inf, loss + tail), 0.0)
    size = size + torch.where(left > 0, left * (left.log().abs() + s_rest.log().abs() + s.log().abs()), 0.0)[:, 0]
    total = p.sum(1, keepdim=True) + left
    q = torch.where(s > 0, e / s, 0.0)
    ratio = torch.where(s_rest > 0, left / s_rest * s, 0.0)
    grad = torch.where(among, q * total, q * (total - ratio)).scatter_add_(1, at, -p)
    f = torch.where(row & ~empty, scale * a[:, 0], 0.0)[:, None]
    reach = torch.where(e > 0, -d, 0.0).clamp(max=100).amax(1, keepdim=True)
    off = 8 * U * (1 + reach) + (cols / 256 + 32) * U
    # p: the exponential of a difference of up to `spread`, over a sum of them
    spread = torch.where(p > 0, log_p.abs(), 0.0).amax(1, keepdim=True) + math.log(value.shape[1])
    off_p = (8 * (1 + spread) + 16) * U
    # each term: p, ln p, the difference and ln S, each off by `off_p`, 4 U of their sizes, and A
    off_loss = (off * total)[:, 0] + (off_p * p.sum(1, keepdim=True))[:, 0] + (16 * U + off_p[:, 0]) * size
    parts = torch.zeros_like(q).scatter_add_(1, at, p)
    off_grad = f.abs() * (2 * (off + 8 * U) * q * (total + torch.where(among, 0.0, ratio)) + (off_p + 4 * U) * parts)
    # (exponentials below the smallest normal number are 0)
    off_grad = off_grad + f.abs() * 2.0 ** -125 * (total / s.clamp(min=1) + torch.where(among | (s_rest == 0), 0.0, left / s_rest.clamp(min=2.0 ** -126)))
    loss, off_loss = [torch.where(torch.isfinite(loss), t, u) for t, u in ((loss, loss), (off_loss, 0.0 * row))]
    return [t.cuda() for t in (loss, off_loss, grad * f, off_grad)]


def teacher(rows, cols, top, seed, rest, dtype=torch.float32, bits=torch.int64):
    gen = generator(seed)
    token = torch.stack([torch.randperm(cols, generator=gen, device="cuda")[:top] if cols >= top else torch.randint(0, cols, (top,), generator=gen, device="cuda")
                         for _ in range(rows)])
    value = 2 * randn((rows, top), torch.float32, seed + 1)
    if rest:                                               # (without all that the rounding to bfloat16 could take above 1)
        value = torch.log_softmax(value, 1) + torch.log1p(-0.02 - 0.5 * torch.rand((rows, 1), generator=gen, device="cuda"))
    if top > 2:
        token[::3, 1], value[::4, 2] = -1, -math.inf       # places that are none
        token[5::7] = -1                                   # and rows of them
        token[6::9, 0] = cols
    return value.to(dtype), token.to(bits)


def check(x, value, token, rest, scale=1.0, teacher_scale=1.0, extra=0, seed=5):
    rows, cols = x.shape
    weight = randn(rows, torch.float32, seed)
    scales = [float(torch.tensor(s)) for s in (scale, teacher_scale)]
    loss, off_loss, grad, off_grad = exact(x, value, token, weight, rest, *scales)
    plan = solo.SoloDistill(rows + 1, cols, value.shape[1], rest=rest, scale=scale, teacher_scale=teacher_scale)
    within(plan.forward(x, value, token), loss, 1.01 * off_loss + 2.0 ** -126)
    first = plan.forward(x, value, token).clone()
    off_grad = 1.01 * (off_grad + ROUND[x.dtype] * (grad.abs() + off_grad)) + 2.0 ** -126
    for call in ("two", "one"):
        whole = torch.full((rows, cols + extra), 7.0, dtype=x.dtype, device="cuda")
        out = whole[:, extra:]
        if call == "two":
            assert plan.grad(x, value, token, weight, out) is out
        else:
            again, got = plan.forward_grad(x, value, token, weight, out)
            assert got is out
            within(again, loss, 1.01 * off_loss + 2.0 ** -126)
        within(out, grad, off_grad)
        assert bool((whole[:, :extra] == 7.0).all())
    over = x.clone()                                       # in place
    plan.forward_grad(over, value, token, weight, over)
    assert torch.equal(over, out)
    return plan, first


# (rows, columns, elements between two rows, alternatives): both sides of every line of the dispatch
SHAPES = [(1, 1, 0, 1), (5, 3, 0, 7), (9, 8, 1, 3), (20, 100, 3, 5), (33, 1000, 0, 20), (12, 2047, 1, 64), (6, 2056, 0, 65), (4, 5000, 0, 128), (5, 8190, 0, 32),
          (3, 9000, 0, 1), (140, 8300, 5, 20), (3, 16390, 0, 33), (4, 32000, 0, 20), (2, 32777, 8, 20), (3, 50257, 47, 32), (2, 65536, 0, 64), (2, 65545, 0, 20), (3, 100_000, 1, 128)]


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,cols,extra,top", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_loss_and_gradient(dtype, rows, cols, extra, top, rest):
    kind = (rows + cols + top) % 2
    value, token = teacher(rows, cols, top, 3, rest, TYPES[kind], (torch.int64, torch.int32)[kind])
    check(strided(rows, cols, dtype, 1, extra, 3.0), value, token, rest, scale=(1.0, 0.5)[kind], teacher_scale=1.0 if rest else 1.7, extra=extra)


# sets on both sides of the lines that go by bytes, for each number of threads that a row can have
MANY = [(40_000, 300), (200, 40_000)] + [(millions * 10 ** 6 // cols, cols) for cols in (1000, 5000, 12_000, 30_000, 60_000, 100_000) for millions in (20, 160)] + [(100, 1_500_000)]


@pytest.mark.parametrize("rows,cols", MANY[:2])
@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows(dtype, rows, cols):
    """Gradients that are written past the caches."""
    gen = generator(3)
    token = torch.randint(0, cols, (rows, 9), generator=gen, device="cuda")
    value = torch.log_softmax(randn((rows, 9), torch.float32, 4), 1) - 0.1
    check(randn((rows, cols), dtype, 1, 2.0), value, token, True)


@pytest.mark.parametrize("rows,cols", MANY[2:])
@pytest.mark.parametrize("dtype", TYPES)
def test_sets_that_are_larger_than_the_caches(dtype, rows, cols):
    """Past the caches, whole sets against the same rows in parts that are not."""
    gen = generator(3)
    x = torch.randn((rows, cols), generator=gen, device="cuda", dtype=dtype)
    token = torch.randint(0, cols, (rows, 5), generator=gen, device="cuda")
    value, weight = torch.log_softmax(randn((rows, 5), torch.float32, 4), 1) - 0.1, torch.rand(rows, generator=gen, device="cuda")
    plan, part = solo.SoloDistill(rows, cols, 5, rest=True), solo.SoloDistill(100, cols, 5, rest=True)
    loss, one = plan.forward(x, value, token).clone(), torch.empty_like(x)
    two = plan.grad(x, value, token, weight, torch.empty_like(x))
    again, _ = plan.forward_grad(x, value, token, weight, one)
    for a in (0, (rows - 100) // 2, rows - 100):
        rows_ = slice(a, a + 100)
        some = x[rows_], value[rows_], token[rows_]
        # (another number of threads may take a row: sums in another order)
        within(loss[rows_], part.forward(*some), 1e-5 * loss[rows_].abs())
        within(again[rows_], part.loss, 1e-5 * loss[rows_].abs())
        small = part.forward_grad(*some, weight[rows_], torch.empty_like(x[rows_]))[1].double()
        for whole in (one, two):
            within(whole[rows_], small, (2 * ROUND[dtype] + 1e-5) * small.abs() + 1e-7)
    for whole in (one, two):                               # the gradient of the shares sums to nothing: every element of every row has been written
        total = whole.double().sum(1)
        within(total, 0 * total, (ROUND[dtype] + 1e-5) * whole.double().abs().sum(1) + 1e-7)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [70, 9000, 70_000])
def test_a_column_that_occurs_twice_and_all_in_one_group(dtype, cols):
    x = randn((6, cols), dtype, 1, 2.0)
    value = torch.log_softmax(randn((6, 40), torch.float32, 2), 1) - 0.2
    for token in (torch.full((6, 40), cols - 1, device="cuda"), torch.arange(40, device="cuda").repeat(6, 1) // 3 + 5, torch.arange(40, device="cuda").repeat(6, 1).flip(1)):
        for rest in (False, True):
            check(x, value, token, rest)


@pytest.mark.parametrize("dtype", TYPES)
def test_masked_students(dtype):
    """-inf in places: beside the alternatives, among them (loss +inf), everywhere; all there is among the alternatives."""
    x = randn((8, 500), dtype, 1, 2.0)
    value, token = torch.log_softmax(randn((8, 6), torch.float32, 2), 1) - 0.1, torch.arange(6, device="cuda").repeat(8, 1) * 80
    x[0, 81:] = -math.inf
    x[1, 160] = -math.inf
    x[2] = -math.inf
    x[3, token[3]] = -math.inf
    x[4] = torch.where(torch.zeros(500, device="cuda").scatter_(0, token[4], 1.0) > 0, x[4], -math.inf)
    x[5] = torch.finfo(dtype).min
    x[6, 7] = 60.0                                         # (the rest is all there is)
    for rest in (False, True):
        plan, loss = check(x, value, token, rest)
        assert loss[1:4].tolist() == [math.inf] * 3 and bool(torch.isfinite(loss[5:]).all())
        assert (loss[4].item() == math.inf) == rest


@pytest.mark.parametrize("cols", [5, 2000, 33_000, 66_000])
def test_a_rest_that_is_small(cols):
    """A student that is sure of an alternative: what is left has all its digits.  And a teacher that leaves less than 2^-20, or nothing."""
    x = randn((3, cols), torch.float32, 1)
    x[:, 2] = torch.tensor([30.0, 60.0, 85.0], device="cuda")
    token = torch.tensor([[2, 3]], device="cuda").repeat(3, 1)
    p = torch.tensor([[0.9, 0.05], [0.5, 0.5 - 2.0 ** -22], [0.75, 0.25]], device="cuda", dtype=torch.float64)
    check(x, p.log().float(), token, True)


def test_a_number_that_is_none_stays_in_its_row():
    x = randn((7, 3000), torch.float32, 1)
    value, token = torch.log_softmax(randn((7, 5), torch.float32, 2), 1) - 0.1, torch.arange(5, device="cuda").repeat(7, 1) * 500
    plan, weight = solo.SoloDistill(7, 3000, 5, rest=True), torch.ones(7, device="cuda")
    loss, grad = [t.clone() for t in plan.forward_grad(x, value, token, weight, torch.empty_like(x))]
    bad, bad_value = x.clone(), value.clone()
    bad[0, 1], bad[2, 500], bad[3, 2999], bad_value[5, 2] = math.nan, math.nan, math.inf, math.nan
    got, got_grad = plan.forward_grad(bad, bad_value, token, weight, torch.empty_like(x))
    assert bool(got[[0, 2, 3, 5]].isnan().all()) and torch.equal(got[[1, 4, 6]], loss[[1, 4, 6]]) and torch.equal(got_grad[[1, 4, 6]], grad[[1, 4, 6]])


def test_rows_without_a_teacher_are_not_read():
    x = torch.full((3, 2500), math.nan, dtype=torch.bfloat16, device="cuda")
    value, token = torch.full((3, 4), math.nan, device="cuda"), torch.full((3, 4), -1, device="cuda")
    token[1], value[1] = 7, -math.inf
    plan, out = solo.SoloDistill(3, 2500, 4), torch.full_like(x, 7.0)
    assert plan.forward(x, value, token).tolist() == [0, 0, 0]
    assert int(plan.grad(x, value, token, torch.ones(3, device="cuda"), out).count_nonzero()) == 0
    assert int(plan.forward_grad(x, value, token, torch.ones(3, device="cuda"), out.fill_(7.0))[1].count_nonzero()) == 0


def test_gradient_against_differences():
    """Every derivative by differences of the 64-bit loss (steps of 1e-4: third derivatives are below 1, so 1e-8, and the call's own bound)."""
    x = randn((2, 12), torch.float32, 1)
    value, token = torch.log_softmax(randn((2, 4), torch.float32, 2), 1) - 0.3, torch.tensor([[3, 9, 3, 0], [11, -1, 5, 6]], device="cuda")
    one = torch.ones(2, device="cuda")
    for rest in (False, True):
        got = solo.SoloDistill(2, 12, 4, rest=rest, scale=0.7).forward_grad(x, value, token, one, torch.empty_like(x))[1]
        for i in range(24):
            ends = []
            for step in (1e-4, -1e-4):
                moved = x.double()
                moved.view(-1)[i] += step
                ends.append(float(exact(moved, value, token, one, rest, float(torch.tensor(0.7)), 1.0)[0].sum()))
            assert abs((ends[0] - ends[1]) / 2e-4 - float(got.view(-1)[i])) < 3e-6, (rest, i)


def test_the_teacher_is_what_its_log_probabilities_return():
    """A teacher's logits, its alternatives, the student's loss: with all columns as alternatives, the divergence of two softmaxes."""
    for cols, top in ((30, 32), (5000, 20)):
        teacher_logits, x = randn((50, cols), torch.bfloat16, 1, 2.0), randn((50, cols), torch.bfloat16, 2, 2.0)
        value, token = solo.SoloLogprob(50, cols, top=top).forward(teacher_logits, None)[-2:]
        plan, loss = check(x, value, token, True)
        if cols <= top:
            p, q = torch.log_softmax(teacher_logits.double(), 1), torch.log_softmax(x.double(), 1)
            within(loss, (p.exp() * (p - q)).sum(1), 1e-4)         # (30 columns of magnitude up to 10, U each: far below)


def test_fewer_rows_and_other_scales():
    x = randn((20, 600), torch.float32, 1)
    value, token = torch.log_softmax(randn((20, 3), torch.float32, 2), 1), torch.arange(3, device="cuda").repeat(20, 1)
    plan, weight = solo.SoloDistill(20, 600, 3), torch.ones(20, device="cuda")
    all_rows = plan.forward(x, value, token).clone()
    assert torch.equal(plan.forward(x[:7], value[:7], token[:7]), all_rows[:7])
    with pytest.raises(ValueError):
        plan.grad(x, value, token, weight, torch.empty_like(x))
    plan.forward(x, value, token)
    plan.scale = 0.5
    with pytest.raises(ValueError):
        plan.grad(x, value, token, weight, torch.empty_like(x))
    none = plan.forward(x[:0], value[:0], token[:0])
    assert none.shape == (0,)


def test_in_a_graph():
    x = randn((40, 9000), torch.bfloat16, 1)
    value, token = torch.log_softmax(randn((40, 20), torch.float32, 2), 1) - 0.1, torch.randint(0, 9000, (40, 20), device="cuda")
    weight, out = torch.rand(40, device="cuda"), [torch.empty_like(x) for _ in range(2)]
    plan, other = solo.SoloDistill(40, 9000, 20, rest=True), solo.SoloDistill(40, 9000, 20, rest=True)

    def run(p, to):
        loss = p.forward(x, value, token)
        p.grad(x, value, token, weight, to[0])
        return loss, p.forward_grad(x, value, token, weight, to[1])[1], to[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(plan, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(plan, out)
    for k in range(3):
        x.copy_(randn((40, 9000), torch.bfloat16, 10 + k))
        token.copy_(torch.randint(0, 9000, (40, 20), generator=generator(k), device="cuda"))
        graph.replay()
        eager = run(other, [torch.empty_like(x) for _ in range(2)])
        torch.cuda.synchronize()
        assert all(torch.equal(a, e) for a, e in zip(got, eager))
