"""Log probability and entropy of rows whose target has nearly all of the probability, against 64 bits.

The target is the last of two logits that one thread of the kernel sees, 4.5 to 5.5 above the first; nothing else counts.  With sums relative to the
largest logit, S = 1 + f with f = e^-5.5 .. e^-4.5 < 0.012, logprob = -ln S and entropy = ln S + f d / S, d < 5.5.  u = 2^-24:

  f      two roundings of the exponent (8 binary orders: 16 u ln 2), 2 u of the exponential: 14 u of itself, below 0.2 u
  S      its sum's rounding: u
  ln S   an error of S of 1.2 u; the logarithm's own, in the last place of a value below 0.02, or 2 u near 1
  f d    14 u + 4 u of 0.012 * 5.5 = 0.066: 1.2 u
"""
import math

import pytest
import torch

from paper_2505_00347_amd import solo

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,groups", [(3000, 2048, 64), (300, 20_000, 1024), (60, 20_000, 1024), (4100, 16_300, 1024), (300, 70_000, 1024)])
def test_confident_rows(rows, cols, groups, dtype):
    """`groups`: of 16 bytes, a multiple of the threads of a row, so that group 0 and group `groups` are one thread's."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    at = groups * 16 // dtype.itemsize
    first = (torch.randn(rows, generator=gen, device="cuda") * 3).to(dtype)
    last = (first + 4.6 + 0.8 * torch.rand(rows, generator=gen, device="cuda")).to(dtype)
    x = torch.full((rows, cols), -math.inf, dtype=dtype, device="cuda")
    x[:, 0], x[:, at] = first, last
    d = last.double() - first.double()
    assert 4.5 <= float(d.min()) and float(d.max()) <= 5.5
    log_s, f = torch.log1p(torch.exp(-d)), torch.exp(-d)
    want, want_entropy = -log_s, log_s + f * d / (1 + f)
    t, w = torch.full((rows,), at, device="cuda"), torch.ones(rows, device="cuda")
    plan = solo.SoloLogprob(rows, cols, top=1)
    logprob, entropy, value, token = plan.forward(x, t)
    again, entropy_again, _ = solo.SoloLogprob(rows, cols).forward_grad(x, t, w, None, torch.empty_like(x))
    for got in (logprob, value[:, 0], again):
        assert float((got.double() - want).abs().max()) <= 4 * U
        assert bool((got <= 0).all())
    for got in (entropy, entropy_again):
        assert float((got.double() - want_entropy).abs().max()) <= 6 * U
    assert bool((token[:, 0] == at).all())
