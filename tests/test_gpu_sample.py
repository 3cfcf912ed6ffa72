"""Sampling on the GPU against a plain implementation in 64 bits.

Tokens have to be equal.  Both sides compare running sums with a goal: the kernel's weights are whole multiples of 2^-shift of the largest and
off by 4e-14 of themselves, so a sum of all columns is off by at most cols * 2^-(shift + 1) + 4e-14 of itself; a row in which a goal lies nearer to a border than
that (and 1e-12 for the sums in 64 bits) says nothing and is left out, unless its sums are whole numbers and exact on both sides."""
import math

import pytest
import torch

from paper_2505_00347_amd import solo
from test_gpu_operators import TYPES, U, generator, randn, strided, within

pytestmark = pytest.mark.gpu


def exact(x, u, temperature, top_k, top_p, min_p):
    """Token, log probability and whether the row is clear of borders."""
    x, (rows, cols) = x.double(), x.shape
    t, p, m, u = (v.double()[:, None] for v in (temperature, top_p, min_p, u.clamp(0, 1 - 2.0 ** -24)))
    k = torch.where(top_k > 0, top_k.long(), cols)[:, None]
    most = x.amax(1, keepdim=True)
    w = torch.where(t > 0, ((x - most) / torch.where(t > 0, t, 1.0)).exp(), (x == most).double())
    w = torch.where(x == most, 1.0, torch.where(x > -math.inf, w, 0.0))
    k = torch.where(t > 0, k, 1)
    order = x.sort(dim=1, descending=True, stable=True).indices
    w = w.gather(1, order)
    shift = min(51, 62 - max(0, math.ceil(math.log2(cols))))
    off = cols * 2.0 ** -(shift + 1) + 2e-12
    clear = torch.where((m > 0) & (m < 1), (w - m).abs() > 1e-12, True).all(1)
    first = (torch.arange(cols, device=x.device) < k) & (w >= m.clamp(max=1))
    w = torch.where(first, w, 0.0)
    sums = w.cumsum(1)
    goal = p.clamp(min=0) * sums[:, -1:]
    clear &= torch.where((p > 0) & (p < 1), ((sums - goal).abs() > 2 * off * sums[:, -1:]) | (w == 0), True).all(1)
    before = torch.cat([torch.zeros_like(goal), sums[:, :-1]], 1)
    first = (p >= 1) | (before < goal)
    first[:, 0] = True
    w = torch.where(first, w, 0.0)
    sums = w.cumsum(1)
    mass = sums[:, -1:]
    clear &= torch.where((u * mass > 0) & (sums < mass), (sums - u * mass).abs() > 2 * off * mass, True).all(1)
    at = (sums > u * mass).int().argmax(1, keepdim=True)
    # (from the logits: a weight has lost what is below the smallest number)
    logprob = torch.where(t > 0, (x.gather(1, order.gather(1, at)) - most) / torch.where(t > 0, t, 1.0) - mass.log(), 0.0)
    return order.gather(1, at)[:, 0], logprob[:, 0], clear, off


def check(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, least_clear=0.98, exact_sums=False):
    rows, cols = x.shape
    named = dict(temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    own = {n: v for n, v in named.items() if isinstance(v, torch.Tensor)}
    plan = solo.SoloSampler(rows + 1, cols, **{n: v for n, v in named.items() if n not in own})
    token, logprob = plan.sample(x, u, **own)
    full = {n: v if n in own else torch.full((rows,), v, device="cuda", dtype=torch.int32 if n == "top_k" else torch.float32) for n, v in named.items()}
    want, want_logprob, clear, off = exact(x, u, **full)
    if exact_sums:
        clear = torch.ones_like(clear)
    assert float(clear.double().mean()) >= least_clear
    bad = torch.nonzero(clear & (token != want))[:5, 0].tolist()
    assert not bad, [(r, int(token[r]), int(want[r]), float(logprob[r]), float(want_logprob[r])) for r in bad]
    within(logprob[clear], want_logprob[clear], 2 * U * want_logprob[clear].abs() + 2 * off)
    # parameters of the rows' own and of all rows give the same
    again = solo.SoloSampler(rows, cols).sample(x, u, **full)
    assert torch.equal(again[0], token) and torch.equal(again[1].nan_to_num(7.0), logprob.nan_to_num(7.0))
    return token, logprob


def uniform(rows, seed):
    return torch.rand(rows, generator=generator(seed), device="cuda")


SHAPES = [(1, 1, 0), (9, 2, 0), (50, 7, 1), (300, 100, 0), (64, 1000, 3), (1100, 1500, 0), (20, 4096, 0), (9, 8192, 0), (9, 8193, 1), (9, 16_390, 0), (300, 15_000, 0),
          (300, 20_000, 0), (270, 33_000, 0), (20, 15_000, 0), (3, 25_000, 0), (6, 32_000, 0), (5, 50_257, 47),
          (3, 65_540, 0), (2, 150_001, 0), (2100, 700, 0), (2100, 1500, 1), (1030, 13_000, 0)]

PARAMETERS = [dict(), dict(temperature=0.0), dict(temperature=0.7, top_p=0.9), dict(top_k=1), dict(top_k=40), dict(top_k=1500, temperature=1.5), dict(min_p=0.05),
              dict(top_k=50, top_p=0.8, min_p=0.01, temperature=1.3), dict(top_p=0.3, min_p=0.2), dict(top_k=7, min_p=1.0)]


@pytest.mark.parametrize("parameters", PARAMETERS, ids=lambda p: "-".join("%s%g" % i for i in p.items()) or "plain")
@pytest.mark.parametrize("rows,cols,extra", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_tokens(dtype, rows, cols, extra, parameters):
    check(strided(rows, cols, dtype, rows + cols, extra, 3.0), uniform(rows, cols), **parameters)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [500, 20_000])
def test_rows_with_parameters_of_their_own(dtype, cols):
    rows = 240
    i = torch.arange(rows, device="cuda")
    choose = lambda values, every: torch.tensor(values, device="cuda")[i // every % len(values)]     # noqa: E731
    check(randn((rows, cols), dtype, 1, 2.5), uniform(rows, 2), temperature=choose([1.0, 0.0, 0.4, 2.0], 1), top_k=choose([0, 5, 300, -1, 10 ** 9], 4).int(),
          top_p=choose([1.0, 0.9, 0.2, 0.0, 7.0], 20), min_p=choose([0.0, 0.1, -1.0], 80))
    check(randn((rows, cols), dtype, 3, 2.5), uniform(rows, 4), temperature=0.8, top_p=choose([1.0, 0.5], 1), top_k=30)


@pytest.mark.parametrize("cols", [900, 6000, 30_000])
@pytest.mark.parametrize("spread", [0.0, 0.01, 0.5, 30.0])
@pytest.mark.parametrize("dtype", TYPES)
def test_flat_and_peaked_rows(dtype, spread, cols):
    """Thousands of equal logits (bfloat16 has few values near each other), a nucleus of most of the row, one of a single column."""
    x = randn((12, cols), dtype, 1, spread) + 5
    for parameters in (dict(), dict(top_p=0.95), dict(top_k=2000), dict(top_k=5000, top_p=0.7, temperature=2.0), dict(min_p=0.5), dict(temperature=0.05, top_p=0.99)):
        if spread:
            check(x, uniform(12, 2), least_clear=0.5, **parameters)
        else:
            check(x, uniform(12, 2), exact_sums=True, **{**parameters, "top_p": 0.5 if "top_p" in parameters else 1.0})


@pytest.mark.parametrize("parameters", [{}, dict(top_p=0.9), dict(top_p=0.7, top_k=37), dict(top_k=3000)], ids=lambda p: "-".join("%s%g" % i for i in p.items()) or "min_p")
@pytest.mark.parametrize("cols", [900, 6000, 30_000, 60_000])
@pytest.mark.parametrize("dtype", TYPES)
def test_numbers_of_columns_above_a_bound(dtype, cols, parameters):
    """min_p keeps n columns of a row exactly, for n on both sides of what is put in order at once and of what a list holds."""
    counts = torch.tensor([n for n in (1, 2, 63, 64, 65, 127, 128, 129, 512, 513, 1023, 1024, 1025, 2048, 2049, 4095, 4096, 4097, 20_000) if n <= cols], device="cuda")
    place = torch.rand(len(counts), cols, generator=generator(70), device="cuda").argsort(1)
    x = 2 * torch.rand(len(counts), cols, generator=generator(71), device="cuda") - 1      # (no w of these is below e^-2)
    x = torch.where(place < counts[:, None], x, x - 20).to(dtype)
    check(x, uniform(len(counts), 72), min_p=0.1, least_clear=0.9, **parameters)


def test_equal_logits_go_by_the_column():
    """n equal columns: the token is column floor(u n) of those that are kept, exactly."""
    for cols in (8, 1024, 1025, 4096, 65_536, 100_000):
        # (half of an odd number: the sum of (cols + 1) / 2 ones is the first that reaches it)
        for kept, parameters in ((cols, {}), ((cols + 1) // 2, dict(top_p=0.5)), (cols // 4, dict(top_k=cols // 4)), (cols // 8, dict(top_k=cols // 4, top_p=0.5)), (1, dict(top_p=0.0)), (1, dict(top_k=1)), (1, dict(temperature=0.0)),
                                 (cols, dict(min_p=1.0)), (cols // 2, dict(min_p=0.5, top_k=cols // 2))):
            u = torch.tensor([0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24], device="cuda")
            x = torch.full((5, cols), -3.0, device="cuda")
            token, logprob = solo.SoloSampler(5, cols, **parameters).sample(x, u)
            assert token.tolist() == [math.floor(float(v) * kept) for v in u], (cols, parameters)
            within(logprob, torch.full((5,), -math.log(kept), dtype=torch.float64, device="cuda"), 2 * U * math.log(kept))


@pytest.mark.parametrize("cols", [1000, 8000, 90_000])
def test_few_values_in_a_row(cols):
    x = torch.randint(0, 4, (16, cols), generator=generator(1), device="cuda").float() * 0.5
    for parameters in (dict(), dict(top_p=0.6), dict(top_k=cols // 3), dict(top_k=100, top_p=0.5), dict(min_p=0.5, top_p=0.9)):
        ones = parameters.get("top_k") == 100              # (more than 100 columns have the largest value)
        check(x, uniform(16, 2), least_clear=0.8, exact_sums=ones, **parameters)
        check(x.bfloat16(), uniform(16, 3), least_clear=0.8, exact_sums=ones, **parameters)


def test_every_column_gets_its_share():
    """4096 evenly spaced numbers on one row: each column as often as its probability says, within one."""
    x = randn((1, 50), torch.float32, 1, 1.5)
    n = 4096
    token, _ = solo.SoloSampler(n, 50, temperature=0.9).sample(x.expand(n, 50).contiguous(), (torch.arange(n, device="cuda") + 0.5) / n)
    share = torch.softmax(x[0].double() / 0.9, 0) * n
    assert bool(((torch.bincount(token, minlength=50) - share).abs() <= 1 + 1e-3).all())


def test_numbers_at_and_beyond_the_ends():
    x = randn((6, 3000), torch.float32, 1)
    u = torch.tensor([0.0, -0.0, -1.0, 1.0, 5.0, math.inf], device="cuda")
    token, _ = check(x, u)
    largest, smallest = x.argmax(1), x.argmin(1)
    assert torch.equal(token[:3], largest[:3]) and torch.equal(token[3:], smallest[3:])


@pytest.mark.parametrize("temperature", [1e-45, 1e-30, 1e-3, 1e4, 1e30, math.inf])
def test_temperatures_at_the_ends(temperature):
    x = randn((8, 2000), torch.float32, 1)
    x[:, 70] = x[:, 7] = 9.0                               # the maximum twice
    x[3, 5:] = -math.inf
    t = torch.full((8,), temperature, device="cuda")
    if temperature >= 1e30:                                # every weight is 1
        check(x, uniform(8, 2), temperature=t, exact_sums=True)
        token, logprob = solo.SoloSampler(8, 2000, temperature=temperature).sample(x, uniform(8, 2))
        assert token[3].item() == torch.argsort(x[3, :5], descending=True, stable=True)[int(uniform(8, 2)[3] * 5)].item()
    else:
        token, logprob = check(x, uniform(8, 2), temperature=t, exact_sums=temperature < 1e-20)
    if temperature < 1e-20:
        assert set(token[[0, 1, 2, 4, 5, 6, 7]].tolist()) <= {7, 70}


@pytest.mark.parametrize("cols", [9, 300, 20_000])
@pytest.mark.parametrize("dtype", TYPES)
def test_masked_rows(dtype, cols):
    x = randn((7, cols), dtype, 1, 2.0)
    x[0, 1:] = -math.inf
    x[1, :-1] = -math.inf
    x[2, ::2] = -math.inf
    x[3] = -math.inf
    x[4, 3] = math.nan
    x[5, 4] = math.inf
    x[6] = torch.finfo(dtype).min
    for parameters in (dict(), dict(top_k=2), dict(top_p=0.5), dict(temperature=0.0), dict(min_p=0.1, top_k=3, top_p=0.9)):
        token, logprob = solo.SoloSampler(7, cols, **parameters).sample(x, uniform(7, 2))
        assert token[:2].tolist() == [0, cols - 1] and logprob[:2].tolist() == [0, 0]
        assert token[2].item() % 2 == 1
        assert token[3:6].tolist() == [-1] * 3 and logprob[3].item() == -math.inf and bool(logprob[4:6].isnan().all())
        good = torch.tensor([0, 1, 2], device="cuda")
        check(x[good], uniform(7, 2)[good], **parameters)
        assert 0 <= token[6].item() < cols


def test_parameters_that_are_no_numbers():
    x, nan = randn((5, 100), torch.float32, 1), math.nan
    ones = torch.ones(5, device="cuda")
    bad = torch.tensor([1.0, nan, 1.0, -1.0, 1.0], device="cuda")
    token, logprob = solo.SoloSampler(5, 100).sample(x, ones * 0.5, temperature=bad)
    assert token[[1, 3]].tolist() == [-1, -1] and bool(logprob[[1, 3]].isnan().all()) and bool((token[[0, 2, 4]] >= 0).all())
    for name in ("top_p", "min_p"):
        token, logprob = solo.SoloSampler(5, 100).sample(x, ones * 0.5, **{name: torch.tensor([1.0, nan, 0.5, -1.0, 0.5], device="cuda")})
        assert token[1].item() == -1 and bool(logprob[1].isnan()) and bool((token[[0, 2, 3, 4]] >= 0).all())
    assert solo.SoloSampler(5, 100).sample(x, ones * nan)[0].tolist() == [-1] * 5


def test_tokens_of_32_bits_and_without_log_probability():
    x, u = randn((9, 700), torch.float32, 1), uniform(9, 2)
    want = solo.SoloSampler(9, 700, top_p=0.9).sample(x, u)[0]
    token = torch.full((10,), 7, dtype=torch.int32, device="cuda")
    solo.solo_sample(x, u, None, None, None, None, token, None, solo.solo_sample_shape(9, 700, 700, 0, 32, 0, 0, 1.0, 0.9, 0.0, 0))
    assert torch.equal(token[:9].long(), want) and token[9].item() == 7


def test_rows_that_lie_more_than_32_bits_apart():
    stride = (1 << 31) - 8
    buffer = torch.full((2 * stride + 16,), -math.inf, dtype=torch.bfloat16, device="cuda")
    far = buffer.as_strided((3, 16), (stride, 1))
    far.copy_(randn((3, 16), torch.bfloat16, 1))
    plan, u = solo.SoloSampler(3, 16), uniform(3, 2)
    want = plan.sample(far.contiguous(), u)[0].clone()
    assert torch.equal(plan.sample(far, u)[0], want)


def test_fewer_rows_and_other_numbers():
    x, u = randn((50, 400), torch.float32, 1), uniform(50, 2)
    plan = solo.SoloSampler(50, 400)
    want = plan.sample(x, u)[0].clone()
    assert torch.equal(plan.sample(x[:7], u[:7])[0], want[:7]) and plan.sample(x[:0], u[:0])[0].numel() == 0
    plan.temperature = 0.0
    assert torch.equal(plan.sample(x, u)[0], x.argmax(1))


def test_in_a_graph():
    x, u = randn((30, 9000), torch.float32, 1, 2.0), uniform(30, 1)
    k = torch.full((30,), 20, dtype=torch.int32, device="cuda")
    plan, other = solo.SoloSampler(30, 9000, top_p=0.9), solo.SoloSampler(30, 9000, top_p=0.9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plan.sample(x, u, top_k=k)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = plan.sample(x, u, top_k=k)
    for n in range(3):
        x.copy_(randn((30, 9000), torch.float32, 10 + n, 2.0))
        u.copy_(uniform(30, n))
        k.fill_((0, 3, 700)[n])
        graph.replay()
        want = other.sample(x, u, top_k=k)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
