"""Layer norm and its gradient on the GPU against a plain implementation in 64 bits.

Bounds.  U = 2^-24, r: half a step of the output's type (2^-24 or 2^-8).  A thread adds up to 16 elements of a row (cols / 1024 where rows
are longer than 16384), ten steps join the threads and four operations follow: a sum over a row is off by at most k U times the sum of its
terms' absolute values, k = 32 + cols / 1024."""
import math

import pytest
import torch

from paper_2505_00347_amd import solo
from test_gpu_operators import ROUND, TYPES, U, randn, strided, within

pytestmark = pytest.mark.gpu

EPS = 1e-5
PAIRS = [(a, b) for a in TYPES for b in TYPES]
# (rows, columns, elements between two rows): both sides of every line of the dispatch, one column to long rows
SHAPES = [(1, 1, 0), (3, 7, 0), (70, 8, 1), (33, 9, 0), (260, 64, 0), (65, 65, 3), (19, 256, 0), (40, 257, 0), (7, 511, 1), (9, 512, 8), (6, 513, 0),
          (1025, 100, 0), (5, 1000, 0), (4, 1024, 0), (5, 1025, 0), (3, 2056, 5), (2500, 768, 0), (3, 4096, 0), (2, 4097, 1), (3, 8192, 0), (2, 8200, 0),
          (1, 16384, 0), (2, 16385, 0), (3, 20001, 1), (70, 16400, 0)]


def exact(x, w, b, dy, rms, eps=EPS):
    """y, mean, rstd, dx, dw, db and what the bounds are made of, in 64 bits."""
    x, dy = x.double(), dy.double()
    n = x.shape[1]
    w = torch.ones(n, dtype=torch.float64, device=x.device) if w is None else w.double()
    b = torch.zeros(n, dtype=torch.float64, device=x.device) if b is None else b.double()
    mean = torch.zeros_like(x[:, :1]) if rms else x.mean(1, keepdim=True)
    c = x - mean
    rstd = 1 / (c.square().mean(1, keepdim=True) + eps).sqrt()
    h = c * rstd
    y = h * w + b
    g = dy * w
    s1, s2 = g.mean(1, keepdim=True) * (not rms), (g * h).mean(1, keepdim=True)
    dx = rstd * (g - s1 - h * s2)
    k = 32 + n / 1024
    # A first mean m is off by up to o = k U mean|x|.  The differences d = x - m, each off by U |d|, are at most |c| + o; their mean, which is taken
    # out, is off by k U (mean|c| + o), so forward's centre is as well; sum d^2 / n - (sum d / n)^2 is off by 2 k U mean (|c| + o)^2, and the
    # root halves its share of the variance.  The mean that is stored is rounded once more, which the gradient's h sees.
    o = k * U * x.abs().mean(1, keepdim=True) * (not rms)
    off_centre = k * U * (c.abs().mean(1, keepdim=True) + o) * (not rms)
    off_rstd = k * U * (c.abs() + o).square().mean(1, keepdim=True) * rstd.square() + 6 * U
    off_forward = rstd * (2 * U * (c.abs() + o) + off_centre) + h.abs() * off_rstd
    off_y = w.abs() * off_forward + 3 * U * (h * w).abs() + 2 * U * b.abs()
    off_mean = off_centre + 2 * U * mean.abs()
    off_h = rstd * (U * c.abs() + off_mean) + h.abs() * off_rstd
    off_s1 = k * U * g.abs().mean(1, keepdim=True)
    off_s2 = k * U * (g * h).abs().mean(1, keepdim=True) + (g.abs() * off_h).mean(1, keepdim=True)
    off_dx = rstd * (2 * U * g.abs() + off_s1 + h.abs() * off_s2 + off_h * s2.abs() + 3 * U * (g.abs() + s1.abs() + (h * s2).abs())) + dx.abs() * off_rstd
    dw, db = (dy * h).sum(0), dy.sum(0)
    off_dw = (len(x) + 8) * U * (dy * h).abs().sum(0) + (dy.abs() * off_h).sum(0)
    off_db = (len(x) + 8) * U * dy.abs().sum(0)
    return dict(y=(y, off_y), mean=(mean, off_mean), rstd=(rstd, rstd * off_rstd), dx=(dx, off_dx), dw=(dw, off_dw), db=(db, off_db))


def near(got, pair, more=0.0):
    want, off = pair
    within(got, want, 1.01 * (off + ROUND[got.dtype] * (want.abs() + off)) + more + 2.0 ** -133)


def weights(cols, dtype, seed=7):
    return (1 + 0.2 * randn(cols, torch.float32, seed)).to(dtype), (0.3 * randn(cols, torch.float32, seed + 1)).to(dtype)


def check(x, w, b, dy, rms=False, eps=EPS, y_extra=0):
    rows, cols = x.shape
    want = exact(x, w, b, dy, rms, eps=float(torch.tensor(eps)))
    plan = solo.SoloLayerNorm(rows + 2, cols, eps=eps, rms=rms)
    whole = torch.full((rows, cols + y_extra), 7.0, dtype=dy.dtype, device="cuda")
    out = plan.forward(x, w, b, whole[:, y_extra:])
    near(out, want["y"])
    assert bool((whole[:, :y_extra] == 7.0).all())
    near(plan.stats[:rows, :1], want["mean"])
    near(plan.stats[:rows, 1:], want["rstd"])
    weight_dtype = w.dtype if w is not None else torch.float32
    whole = torch.full((rows, cols + y_extra), 7.0, dtype=x.dtype, device="cuda")
    grads = whole[:, y_extra:], *(torch.full((cols,), 7.0, dtype=weight_dtype, device="cuda") for _ in range(2))
    got = plan.grad(dy, x, w, *grads)
    assert got[0] is grads[0] and got[1] is grads[1] and got[2] is grads[2]
    for g, name in zip(got, ("dx", "dw", "db")):
        near(g, want[name])
    assert bool((whole[:, :y_extra] == 7.0).all())
    return plan, want, got


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("rows,cols,extra", SHAPES)
@pytest.mark.parametrize("dtype,out_dtype", PAIRS)
def test_forward_and_gradient(dtype, out_dtype, rows, cols, extra, rms):
    weight_dtype = TYPES[(rows + cols) % 2]
    x = strided(rows, cols, dtype, 1, extra, 2.0) + randn((rows, 1), dtype, 2)
    x = torch.cat([x, x[:, :extra]], 1)[:, :cols] if extra else x
    dy = strided(rows, cols, out_dtype, 3, extra, 0.1)
    w, b = weights(cols, weight_dtype)
    check(x, w, None if rms else b, dy, rms, y_extra=extra)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [9, 300, 768, 3000, 16400])
def test_without_weights_and_one_by_one(dtype, cols):
    """weight and bias None; each gradient by itself is the one of the full call, bit by bit; sums are added where asked."""
    x, dy = randn((50, cols), dtype, 1), randn((50, cols), dtype, 2)
    plan, want, full = check(x, None, None, dy)
    for k in range(3):
        out = [torch.full_like(g, 7.0) if i == k else None for i, g in enumerate(full)]
        assert torch.equal(plan.grad(dy, x, None, *out)[k], full[k])
    old = randn(cols, torch.float32, 3), randn(cols, torch.float32, 4)
    added = [t.clone() for t in old]
    plan.grad(dy, x, None, None, *added, accumulate=True)
    assert all(torch.equal(a, t + g) for a, t, g in zip(added, old, full[1:]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [40, 900, 5000, 17000])
def test_in_place(dtype, cols):
    w, b = weights(cols, dtype)
    x, dy = randn((37, cols), dtype, 1), randn((37, cols), dtype, 2)
    plan = solo.SoloLayerNorm(37, cols)
    y = plan.forward(x, w, b, torch.empty_like(x)).clone()
    want = [g.clone() for g in plan.grad(dy, x, w, torch.empty_like(x), torch.empty_like(w), torch.empty_like(w))]
    for over in (x, dy):                                   # the gradient over either of its inputs
        copies = {id(t): t.clone() for t in (x, dy)}
        got = plan.grad(copies[id(dy)], copies[id(x)], w, copies[id(over)], torch.empty_like(w), torch.empty_like(w))
        assert all(torch.equal(a, c) for a, c in zip(got, want))
    assert torch.equal(plan.forward(x, w, b, x), y)


def test_rows_far_from_zero_and_rows_without_spread():
    """The differences from the mean keep their digits; a constant row is the bias."""
    w, b = weights(1000, torch.float32)
    x = randn((6, 1000), torch.float32, 1) + torch.tensor([0.0, 1e3, -1e5, 1e6, 3e-3, 40.0], device="cuda")[:, None]
    check(x, w, b, randn((6, 1000), torch.float32, 2))
    for value in (0.0, 5.0, -1e30):
        x = torch.full((3, 1000), value, device="cuda")
        y = solo.SoloLayerNorm(3, 1000).forward(x, None, b, torch.empty_like(x))
        within(y, b.expand(3, -1), 32 * 2 * U * abs(value) / math.sqrt(EPS) + 0 * b)
    small = randn((5, 700), torch.float32, 3, 1e-9)        # (eps is all there is)
    check(small, None, None, randn((5, 700), torch.float32, 4), eps=1e-12)


@pytest.mark.parametrize("cols", [5, 64, 200, 600, 2000, 9000, 17000])
def test_a_row_that_is_not_finite_stays_by_itself(cols):
    x, dy = randn((21, cols), torch.bfloat16, 1), randn((21, cols), torch.bfloat16, 2)
    plan = solo.SoloLayerNorm(21, cols)
    y = plan.forward(x, None, None, torch.empty_like(x)).clone()
    dx = plan.grad(dy, x, None, torch.empty_like(x), None, None)[0].clone()
    bad = x.clone()
    bad[4, cols // 2], bad[11, cols - 1] = math.nan, math.inf
    others = [r for r in range(21) if r not in (4, 11)]
    assert torch.equal(plan.forward(bad, None, None, torch.empty_like(x))[others], y[others])
    assert torch.equal(plan.grad(dy, bad, None, torch.empty_like(x), None, None)[0][others], dx[others])
    assert bool(plan.forward(bad, None, None, torch.empty_like(x))[4].isnan().all())
    assert bool(solo.SoloLayerNorm(21, cols, rms=True).forward(bad, None, None, torch.empty_like(x))[4].isnan().all())


def test_fewer_rows_than_the_handle_has_room_for_and_none():
    w, b = weights(48, torch.float32)
    plan = solo.SoloLayerNorm(1000, 48)
    for n in (1000, 1, 63, 0, 257):
        x, dy = randn((n, 48), torch.float32, n + 1), randn((n, 48), torch.float32, n + 2)
        want = exact(x, w, b, dy, False)
        near(plan.forward(x, w, b, torch.empty_like(x)), want["y"])
        for got, name in zip(plan.grad(dy, x, w, *(torch.full_like(t, 7.0) for t in (x, w, b))), ("dx", "dw", "db")):
            near(got, want[name])
    none, old = torch.empty((0, 48), device="cuda"), torch.full((48,), 7.0, device="cuda")
    plan.grad(none, none, w, None, old, None, accumulate=True)
    assert bool((old == 7).all())


def test_gradient_against_differences():
    """Every derivative of a weighted sum of the outputs, by differences of the 64-bit function: off by the third derivative times 1e-8 (steps
    of 1e-4), which is below 1e-5 of the rows' gradients here, and the call's own bound."""
    for rms in (False, True):
        x, dy = randn((2, 9), torch.float32, 1), randn((2, 9), torch.float32, 2)
        w, b = weights(9, torch.float32)
        plan = solo.SoloLayerNorm(2, 9, rms=rms)
        plan.forward(x, w, b, torch.empty_like(x))
        got = plan.grad(dy, x, w, *(torch.empty_like(t) for t in (x, w, b)))
        loss = lambda x, w, b: float((exact(x, w, b, dy, rms)["y"][0] * dy.double()).sum())     # noqa: E731
        inputs = [t.double() for t in (x, w, b)]
        for k, g in enumerate(got):
            for i in range(g.numel()):
                ends = []
                for step in (1e-4, -1e-4):
                    moved = [t.clone() for t in inputs]
                    moved[k].view(-1)[i] += step
                    ends.append(loss(*moved))
                slope = (ends[0] - ends[1]) / 2e-4
                assert abs(slope - float(g.view(-1)[i])) < 2e-5 * (1 + abs(slope)), (rms, k, i)


def test_same_bits_on_every_call():
    x, dy = randn((5000, 776), torch.bfloat16, 1), randn((5000, 776), torch.bfloat16, 2)
    w, b = weights(776, torch.float32)
    plan = solo.SoloLayerNorm(5000, 776)
    plan.forward(x, w, b, torch.empty_like(x))
    first = [g.clone() for g in plan.grad(dy, x, w, *(torch.empty_like(t) for t in (x, w, b)))]
    for _ in range(3):
        again = plan.grad(dy, x, w, *(torch.full_like(t, 7.0) for t in (x, w, b)))
        assert all(torch.equal(a, f) for a, f in zip(again, first))


def test_rows_that_lie_more_than_32_bits_apart():
    stride = (1 << 31) - 8
    buffer = torch.zeros(2 * stride + 24, dtype=torch.bfloat16, device="cuda")
    far = buffer.as_strided((3, 24), (stride, 1))
    far.copy_(randn((3, 24), torch.bfloat16, 1))
    near_, dy = far.contiguous(), randn((3, 24), torch.bfloat16, 2)
    plan = solo.SoloLayerNorm(3, 24)
    want = plan.forward(near_, None, None, torch.empty_like(near_)).clone()
    assert torch.equal(plan.forward(far, None, None, torch.empty_like(near_)), want)
    dx = plan.grad(dy, near_, None, torch.empty_like(near_), None, None)[0].clone()
    assert torch.equal(plan.grad(dy, far, None, far, None, None)[0], dx)
    assert int(buffer.count_nonzero()) <= 72
    plan.forward(near_, None, None, far)
    assert torch.equal(far, want)


def test_in_a_graph():
    """Forward and gradient captured together and replayed on new inputs, with eager calls of another handle in between."""
    x, dy = randn((300, 520), torch.float32, 1), randn((300, 520), torch.float32, 2)
    w, b = weights(520, torch.float32)
    plan, other = solo.SoloLayerNorm(300, 520), solo.SoloLayerNorm(300, 520)
    out = [torch.empty_like(t) for t in (x, x, w, b)]

    def run(p, to):
        p.forward(x, w, b, to[0])
        p.grad(dy, x, w, *to[1:])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(plan, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(plan, out)
    for k in range(3):
        x.copy_(randn((300, 520), torch.float32, 10 + k))
        dy.copy_(randn((300, 520), torch.float32, 20 + k))
        graph.replay()
        eager = [torch.empty_like(t) for t in out]
        run(other, eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, e) for a, e in zip(out, eager))
