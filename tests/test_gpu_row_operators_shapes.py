"""Shapes at the ends of what layer norm, distillation and sampling take: more rows than a launch has workgroups side by side, rows without columns."""
import math

import pytest
import torch

from paper_2505_00347_amd import solo
from test_gpu_operators import TYPES, generator, randn, within

pytestmark = pytest.mark.gpu
MANY = (1 << 20) + 77


def parts():
    """The first rows, those on both sides of the 2^20th, and the last."""
    return [slice(0, 100), slice((1 << 20) - 50, (1 << 20) + 27), slice(MANY - 100, MANY)]


@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_of_many_rows(dtype):
    x, dy = randn((MANY, 12), dtype, 1), randn((MANY, 12), dtype, 2)
    plan, part = solo.SoloLayerNorm(MANY, 12), solo.SoloLayerNorm(100, 12)
    y, dw, db = plan.forward(x, None, None, torch.empty_like(x)), torch.empty(12, device="cuda"), torch.empty(12, device="cuda")
    dx, _, _ = plan.grad(dy, x, None, torch.full_like(x, 7.0), dw, db)
    for rows in parts():
        some = x[rows]
        assert torch.equal(part.forward(some, None, None, torch.empty_like(some)), y[rows])
        assert torch.equal(part.grad(dy[rows], some, None, torch.empty_like(some), None, None)[0], dx[rows])
    # 2^-24 for each of 512 parts' 8 additions a row of a workgroup's share and their sum, and h off by 2^-19 at most
    h = (x.double() - x.double().mean(1, keepdim=True)) * plan.stats[:, 1:].double()
    share = MANY / (512 * 32) + 600
    within(db, dy.double().sum(0), share * 2.0 ** -24 * dy.double().abs().sum(0))
    within(dw, (dy.double() * h).sum(0), (share * 2.0 ** -24 + 2.0 ** -19) * (dy.double().abs() * (h.abs() + 1)).sum(0))


@pytest.mark.parametrize("dtype", TYPES)
def test_distillation_of_many_rows(dtype):
    x = randn((MANY, 12), dtype, 1, 2.0)
    token = torch.randint(0, 12, (MANY, 2), generator=generator(2), device="cuda", dtype=torch.int32)
    value, weight = torch.log_softmax(randn((MANY, 2), torch.float32, 3), 1) - 0.1, torch.rand(MANY, generator=generator(4), device="cuda")
    plan, part = solo.SoloDistill(MANY, 12, 2, rest=True), solo.SoloDistill(100, 12, 2, rest=True)
    loss = plan.forward(x, value, token).clone()
    grad = plan.grad(x, value, token, weight, torch.full_like(x, 7.0))
    again, one = plan.forward_grad(x, value, token, weight, torch.full_like(x, 7.0))
    for rows in parts():
        some = x[rows], value[rows], token[rows]
        assert torch.equal(part.forward(*some), loss[rows])
        assert torch.equal(part.grad(*some, weight[rows], torch.empty_like(x[rows])), grad[rows])
        got = part.forward_grad(*some, weight[rows], torch.empty_like(x[rows]))
        assert torch.equal(got[0], again[rows]) and torch.equal(got[1], one[rows])


@pytest.mark.parametrize("dtype", TYPES)
def test_sampling_of_many_rows(dtype):
    x, u = randn((MANY, 12), dtype, 1, 2.0), torch.rand(MANY, generator=generator(2), device="cuda")
    plan, part = solo.SoloSampler(MANY, 12, top_p=0.9), solo.SoloSampler(100, 12, top_p=0.9)
    plan.token.fill_(-7)
    token, logprob = plan.sample(x, u)
    assert int(token.min()) >= 0 and int(token.max()) < 12
    for rows in parts():
        got = part.sample(x[rows], u[rows])
        assert torch.equal(got[0], token[rows]) and torch.equal(got[1], logprob[rows])


def test_rows_without_columns():
    x, value, token = torch.empty((4, 0), device="cuda"), torch.zeros((4, 3), device="cuda"), torch.zeros((4, 3), dtype=torch.int64, device="cuda")
    one = torch.ones(4, device="cuda")
    plan = solo.SoloDistill(4, 0, 3)
    assert plan.forward(x, value, token).tolist() == [0.0] * 4
    assert plan.grad(x, value, token, one, torch.empty_like(x)).shape == (4, 0)
    assert plan.forward_grad(x, value, token, one, torch.empty_like(x))[0].tolist() == [0.0] * 4
    got, logprob = solo.SoloSampler(4, 0).sample(x, one / 2)
    assert got.tolist() == [-1] * 4 and logprob.tolist() == [-math.inf] * 4
    norm, none = solo.SoloLayerNorm(4, 0), torch.empty(0, device="cuda")
    assert norm.forward(x, none, none, torch.empty_like(x)).shape == (4, 0)
    assert norm.grad(x, x, none, torch.empty_like(x), none, none)[1].numel() == 0


def test_rows_of_one_column():
    """Layer norm of a single element is the bias; one column is always the token; a student of one column is sure."""
    x = randn((70, 1), torch.float32, 1, 100.0)
    w, b = torch.full((1,), 3.0, device="cuda"), torch.full((1,), 0.5, device="cuda")
    plan = solo.SoloLayerNorm(70, 1)
    assert bool((plan.forward(x, w, b, torch.empty_like(x)) == 0.5).all())
    dx, dw, db = plan.grad(torch.ones_like(x), x, w, torch.empty_like(x), torch.empty_like(w), torch.empty_like(b))
    assert not bool(dx.any()) and not bool(dw.any()) and db.item() == 70
    token, logprob = solo.SoloSampler(70, 1, top_p=0.5, top_k=3, min_p=0.1).sample(x, torch.rand(70, device="cuda"))
    assert not bool(token.any()) and not bool(logprob.any())
