"""Sampling at the ends of what its parameters and shapes allow."""
import math

import pytest
import torch

from paper_2505_00347_amd import solo
from test_gpu_operators import TYPES, U, generator, randn

pytestmark = pytest.mark.gpu


def uniform(rows, seed):
    return torch.rand(rows, generator=generator(seed), device="cuda")


@pytest.mark.parametrize("min_p", [1.0 + 2.0 ** -23, 1.5, 3e38, math.inf])
@pytest.mark.parametrize("rows,cols", [(9, 2), (40, 300), (9, 4000), (9, 9000), (300, 20_000), (9, 50_257), (3, 150_000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_a_floor_above_every_weight_keeps_the_first_column(dtype, rows, cols, min_p):
    """No column has a weight of more than 1, and one is kept at least: of several largest logits the lowest column, whatever the other parameters say."""
    x = randn((rows, cols), dtype, 1)
    x[::2] = x[::2].clamp(max=0.0)                         # (half of such a row is its largest)
    x[1] = 2.0
    want = x.double().eq(x.double().amax(1, keepdim=True)).int().argmax(1)
    for other in (dict(), dict(top_p=0.9), dict(top_k=5), dict(temperature=2.0, top_p=0.5, top_k=100), dict(temperature=0.0)):
        token, logprob = solo.SoloSampler(rows, cols, min_p=min_p, **other).sample(x, uniform(rows, 2))
        assert torch.equal(token, want) and not bool(logprob.any()), other
    floors = torch.where(torch.arange(rows, device="cuda") % 3 == 0, min_p, 1.0)
    token, logprob = solo.SoloSampler(rows, cols).sample(x, uniform(rows, 2), min_p=floors)
    assert torch.equal(token[::3], want[::3]) and not bool(logprob[::3].any())
    # a floor of 1 keeps all of the largest
    ties = x.double().eq(x.double().amax(1, keepdim=True)).sum(1)
    assert torch.allclose(logprob.double(), torch.where(floors > 1, 0.0, -ties.double().log()), atol=0, rtol=2.0 ** -23)


@pytest.mark.parametrize("rows,cols", [(9, 2), (40, 300), (9, 4000), (9, 9000), (300, 20_000), (9, 50_257), (3, 150_000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_numbers_from_1_on_count_as_the_one_next_to_1(dtype, rows, cols):
    """Not as a way to the least likely column of all: its share may be far below 2^-24."""
    x = randn((rows, cols), dtype, 1, 3.0) - 40.0
    x[:, cols // 2] = 2.0
    x[1] = 1.0
    last = torch.full((rows,), 1 - 2.0 ** -24, device="cuda")
    for parameters in (dict(), dict(top_p=0.9), dict(top_k=40), dict(top_k=2000), dict(min_p=1e-30), dict(temperature=0.3)):
        plan = solo.SoloSampler(rows, cols, **parameters)
        token, logprob = (t.clone() for t in plan.sample(x, last))
        for beyond in (1.0, 1.5, 2.0, 1e30, math.inf):
            got = plan.sample(x, torch.full_like(last, beyond))
            assert torch.equal(got[0], token) and torch.equal(got[1], logprob), (parameters, beyond)
        assert token[0].item() == cols // 2


# A weight is a whole multiple of 2^-43 of the largest in a row of 2^19 columns; in longer ones of 2^-51 or, where the sum S of all is above 2^9, of no more than S 2^-60.
# A sum of n columns is off by half of that each, and weights in binary64 are off by 2e-13 of themselves.
def sums_are_off_by(n, total, cols):
    return n * (2.0 ** -44 if cols <= 1 << 19 else max(2.0 ** -52, total * 2.0 ** -61)) + 4e-13 * total


@pytest.mark.parametrize("weight", [1.4, 0.45, 40.0, 3e6])
@pytest.mark.parametrize("cols", [600_001, 1 << 21, 4_000_003])
def test_tails_of_many_small_equal_weights(cols, weight):
    """One column of weight 1 and all others of `weight` times what 1 divided by cols^2 is beside 2^-20: each next to nothing, together a share that numbers of 24 bits see."""
    u = torch.tensor([1 - k * 2.0 ** -24 for k in (1, 3, 10, 40)] + [0.5, 0.0], device="cuda")
    x = torch.full((6, cols), math.log(weight * 2.0 ** -20 / cols), device="cuda")
    x[:, cols // 3] = 0.0
    w = float(torch.exp(x[0, 0].double()))
    total = 1 + (cols - 1) * w
    token, logprob = solo.SoloSampler(6, cols).sample(x, u)
    off = sums_are_off_by(cols, total, cols)
    for number, got, log in zip(u.tolist(), token.tolist(), logprob.double().tolist()):
        if got == cols // 3:
            assert 1 > number * total - 2 * off
        else:
            before = 1 + (got - (got > cols // 3)) * w     # (of those in front of it, in the order of the columns)
            assert before <= number * total + 2 * off and before + w > number * total - 2 * off, (number, got)
        want = (0.0 if got == cols // 3 else math.log(w)) - math.log(total)
        assert abs(log - want) <= 2 * U * abs(want) + off / total
    assert token[5].item() == cols // 3 and (not 1 < weight < 100 or len(set(token[:4].tolist())) == 4)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [524_288, 524_289, 2_000_000])
def test_long_rows(dtype, cols):
    """Any token is right whose part of the running sum holds the goal, within what the sums are off by."""
    x, u = randn((5, cols), dtype, 1, 2.0), uniform(5, 2)
    x[3, ::3] = -math.inf
    x[4] = 1.0
    u[0] = 1 - 2.0 ** -24
    for parameters in (dict(), dict(temperature=3.0), dict(top_p=0.9), dict(top_k=100), dict(top_k=cols // 2, temperature=0.5), dict(min_p=0.05), dict(temperature=math.inf)):
        token, logprob = solo.SoloSampler(5, cols, **parameters).sample(x, u)
        for r in range(5):
            v, order = x[r].double().sort(descending=True, stable=True)
            t = parameters.get("temperature", 1.0)
            w = torch.where(v > -math.inf, torch.exp((v - v[0]) / t), 0.0)
            w = w[:parameters.get("top_k", cols)]
            w = w[w >= float(torch.tensor(parameters.get("min_p", 0.0)))]
            sums = w.cumsum(0)
            off, ends = sums_are_off_by(len(w), float(w.sum()), cols), [len(w)]
            if "top_p" in parameters:                      # (the nucleus may end where its goal lies within the error, too)
                goal = float(torch.tensor(parameters["top_p"])) * float(sums[-1])
                ends = [int(torch.searchsorted(sums, goal + d)) + 1 for d in (-2 * off, 0.0, 2 * off)]
            place = int((order == token[r]).nonzero())
            assert place < max(ends) and w[place] > 0
            masses = [float(sums[e - 1]) for e in ends]
            before, upto = float(sums[place] - w[place]), float(sums[place])
            goals = [float(u[r]) * m for m in masses]
            assert before <= max(goals) + 2 * off and upto > min(goals) - 2 * off, (parameters, r)
            logs = [math.log(float(w[place]) / m) for m in masses]
            assert min(logs) - 2 * U * abs(min(logs)) - 2 * off <= float(logprob[r]) <= max(logs) + 2 * U * abs(max(logs)) + 2 * off


def test_very_many_equal_logits():
    """Whole numbers: exact."""
    cols = (1 << 22) + 3
    u = torch.tensor([0.0, 0.3, 0.75, 1 - 2.0 ** -24], device="cuda")
    token, logprob = solo.SoloSampler(4, cols).sample(torch.full((4, cols), -7.5, device="cuda"), u)
    assert token.tolist() == [math.floor(float(v) * cols) for v in u]
    assert bool(((logprob.double() + math.log(cols)).abs() <= 2 * U * math.log(cols)).all())
