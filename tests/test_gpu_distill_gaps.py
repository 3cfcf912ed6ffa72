"""Distillation where the student's alternatives and its other columns lie far apart: what it leaves for the others is far below the smallest
binary32 number beside its largest probability, but the formulas' loss and gradient are ordinary numbers.

Against logarithms in 64 bits.  Bounds, U = 2^-24: an exponential of a difference of d natural units is off by 8 U (1 + d).  The sum R of the others, relative
to their largest, and S of all, relative to the largest of all, add up such (cols / 256 + 32 steps), S also R times the exponential of the gap:
each is off by no more than 2 A, A = 8 U (1 + reach) + (cols / 256 + 32) U, `reach` being the largest difference that counts, 100 at
most (exponentials below 2^-126 are 0).  A gradient is a product of an exponential, one of the gap and a quotient by a sum: 4 A and some roundings.  A loss has
the logarithms' sizes times 16 U beside A."""
import math

import pytest
import torch

from paper_2505_00347_amd import solo
from test_gpu_operators import ROUND, TYPES, U, randn, within

pytestmark = pytest.mark.gpu


def exact(x, p, token, weight, scale):
    """Loss, gradient and bounds for probabilities p at columns `token`, each of which occurs once, and what they leave of 1."""
    z, p, a = x.double() * scale, p.double(), weight.double()[:, None] * scale
    cols = x.shape[1]
    among = torch.zeros_like(z, dtype=torch.bool).scatter_(1, token, True)
    z_rest, z_k = torch.where(among, -math.inf, z), z.gather(1, token)
    top_rest, top = z_rest.amax(1, keepdim=True), z.amax(1, keepdim=True)
    # (the sums relative to the largest: beside 1e30 their logarithms would be lost in 64 bits, too)
    log_s, log_r = torch.logsumexp(z - top, 1, keepdim=True), torch.logsumexp(z_rest - top_rest, 1, keepdim=True)
    left = 1 - p.sum(1, keepdim=True)
    total = p.sum(1, keepdim=True) + left
    gap = top - top_rest
    loss = (p * (p.log() + (top - z_k) + log_s)).sum(1) + (left * (left.log() + gap - log_r + log_s))[:, 0]
    size = (p * (p.log().abs() + top - z_k + log_s)).sum(1) + (left * (left.log().abs() + log_r + gap + log_s))[:, 0]
    q, share = (z - top - log_s).exp(), (z_rest - top_rest - log_r).exp()
    parts = torch.zeros_like(z).scatter_(1, token, p)
    grad = a * torch.where(among, q * total - parts, q * total - left * share)
    reach = torch.maximum((top - z).clamp(max=100).amax(1, keepdim=True), gap.clamp(max=100))
    off = 8 * U * (1 + reach) + (cols / 256 + 32) * U
    off_p = (8 * (1 + p.log().abs().amax(1, keepdim=True)) + 16) * U
    off_loss = 2 * off[:, 0] + off_p[:, 0] * p.sum(1) + (16 * U + off_p[:, 0]) * size
    off_grad = a.abs() * ((4 * off + 16 * U) * (q * total + left * share) + (off_p + 4 * U) * parts + 2.0 ** -125 * (total + left))
    return loss, off_loss, grad, off_grad


def check(x, p, token, scale):
    rows, cols = x.shape
    value, weight = p.log().float(), randn(rows, torch.float32, 5)
    scale = float(torch.tensor(scale))
    loss, off_loss, grad, off_grad = exact(x, value.double().exp(), token, weight, scale)
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(grad).all())
    off_grad = 1.01 * (off_grad + ROUND[x.dtype] * (grad.abs() + off_grad)) + 2.0 ** -126
    plan = solo.SoloDistill(rows, cols, token.shape[1], rest=True, scale=scale)
    within(plan.forward(x, value, token), loss, 1.01 * off_loss)
    two = plan.grad(x, value, token, weight, torch.full_like(x, 7.0))
    within(two, grad, off_grad)
    over = x.clone()
    assert torch.equal(plan.grad(over, value, token, weight, over), two)
    again, one = plan.forward_grad(x, value, token, weight, torch.full_like(x, 7.0))
    within(again, loss, 1.01 * off_loss)
    within(one, grad, off_grad)
    over = x.clone()
    assert torch.equal(plan.forward_grad(over, value, token, weight, over)[1], one)


# the lead of an alternative over the other columns; of another, in another wavefront where there are some; and alternatives below the others
LEADS = [(0, 0), (20, 3), (60, 0), (86, 0), (88, 1), (90, 0), (97, 62), (104, 100), (200, 0), (0, 1000), (1e4, 0), (1e4, 1e4), (-90, -200), (-1e4, 60), (300, 0)]
P = [[0.9, 0.05], [0.5, 0.25], [0.125, 0.75]]


@pytest.mark.parametrize("scale", [1.0, 4.0, 0.25])
@pytest.mark.parametrize("rows,cols", [(15, 5), (15, 300), (15, 5000), (150, 9000), (15, 33_000), (15, 70_000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_alternatives_that_lead(dtype, rows, cols, scale):
    x = randn((rows, cols), torch.float32, 1)
    lead = torch.tensor(LEADS, device="cuda").repeat(rows // 15, 1) / scale
    token = torch.tensor([[1, cols - 1]], device="cuda").repeat(rows, 1)
    check(x.scatter_add(1, token, lead).to(dtype), torch.tensor(P, device="cuda", dtype=torch.float64).repeat(rows // 3, 1), token, scale)


@pytest.mark.parametrize("masked", [-1e4, -3e4, -1e30])
@pytest.mark.parametrize("cols", [40, 3000, 20_000, 80_000])
@pytest.mark.parametrize("dtype", TYPES)
def test_columns_masked_by_a_large_finite_number(dtype, cols, masked):
    """All but the alternatives (the loss has the mask in it, the gradient of a masked column is its share of what the teacher leaves), or all but some more."""
    x = randn((6, cols), torch.float32, 1)
    token = torch.arange(3, device="cuda").repeat(6, 1) * (cols // 3) + 1
    kept = torch.zeros_like(x).scatter_(1, token, 1.0) > 0
    kept[3:, ::7] = True
    x = torch.where(kept, x, masked).to(dtype)
    check(x, torch.tensor([[0.5, 0.2, 0.1]], device="cuda", dtype=torch.float64).repeat(6, 1), token, 1.0)


def test_the_gradient_sums_to_nothing_and_is_that_of_the_loss():
    """Differences of the 64-bit loss at a lead of 150: steps of 1e-3, third derivatives below 1 (2e-7), and the call's own bound: the others lie within 4 of their
    largest, so A is below 8 U 5 + 33 U, and the gradient off by (4 A + 16 U) times shares of 1.2 in all."""
    x = randn((1, 9), torch.float32, 1)
    x[0, 4] += 150.0
    token, p, one = torch.tensor([[4, 7]], device="cuda"), torch.tensor([[0.7, 0.1]], device="cuda", dtype=torch.float64), torch.ones(1, device="cuda")
    value = p.log().float()
    p = value.double().exp()
    got = solo.SoloDistill(1, 9, 2, rest=True).forward_grad(x, value, token, one, torch.empty_like(x))[1].double()
    within(got.sum(1), torch.zeros(1, device="cuda"), 1.2 * 308 * U)
    for i in range(9):
        ends = []
        for step in (1e-3, -1e-3):
            moved = x.double()
            moved[0, i] += step
            ends.append(float(exact(moved, p, token, one, 1.0)[0]))
        assert abs((ends[0] - ends[1]) / 2e-3 - float(got[0, i])) < 1.2 * 308 * U + 2e-7, i
