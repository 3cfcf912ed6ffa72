"""The operators around the step on the GPU against plain implementations in 64 bits: global norm and clipping, embedding and its
gradient, log probabilities and their gradient.

Bounds.  u = 2^-24 is half the distance from 1 to the next binary32 value, r the relative error of rounding to the output's type
(u, or 2^-8 for bfloat16, which has 8 significant bits).  Each bound is stated where it is used, from the number of roundings on the way to the value."""
import math

import pytest
import torch

from paper_2505_00347_amd import solo

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]
ROUND = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
TINY = 2.0 ** -126


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=generator(seed), device="cuda") * scale).to(dtype)


def within(got, want, bound):
    got, want = got.double(), want.double()
    off = (got - want).abs()
    off = torch.where(got == want, 0.0, off)               # (infinities)
    off = torch.where(got.isnan() & want.isnan(), 0.0, off)
    assert bool((off <= bound).all()), (float(off.max()), int((~(off <= bound)).sum()), off.numel())


# ---- norm and clipping -----------------------------------------------------------------------

def tensors(sizes, types, seed, scale=1e-3):
    """Gradients that begin at odd places of a packed buffer."""
    grads = []
    for k, n in enumerate(sizes):
        dtype = types[k % len(types)]
        flat = randn(n + 3, dtype, seed + k, scale)
        grads.append(flat[k % 4:][:n])
    return grads


def exact_norm(grads, u=1.0):
    squares = [float(g.double().square().sum()) for g in grads]
    return math.sqrt(sum(squares)) * abs(u), [math.sqrt(s) * abs(u) for s in squares]


SETS = [[1], [7], [8], [4096], [16384], [16385], [1, 0, 3, 100_003, 0, 16384 * 3 + 5], [5] * 300, [70_001, 2048 * 8 - 1, 2048 * 8 * 2 + 9]]


@pytest.mark.parametrize("types", [[torch.float32], [torch.bfloat16], TYPES], ids=["fp32", "bf16", "both"])
@pytest.mark.parametrize("sizes", SETS, ids=lambda s: "%dx%d" % (len(s), max(s)))
@pytest.mark.parametrize("unscale", [None, 0.25, -3.0])
def test_norm_and_clip(sizes, types, unscale):
    grads = tensors(sizes, types, len(sizes))
    clipped = [torch.full_like(g, 7.0) for g in grads]
    u = 1.0 if unscale is None else unscale
    want, each = exact_norm(grads, u)
    plan = solo.SoloGradNorm(grads, clipped)
    scale_of = torch.tensor([unscale], device="cuda") if unscale is not None else None
    for max_norm in (want / 2, want * 2, math.inf, 0.0):
        # binary64 sums of exact squares, one rounding to binary32, and u itself exact: 2 u
        norm, scale, tensor_norm = plan.norm(max_norm, scale_of)
        within(norm, torch.tensor([want], device="cuda"), 2 * U * want)
        within(tensor_norm, torch.tensor(each, device="cuda", dtype=torch.float64), 2 * U * torch.tensor(each, device="cuda", dtype=torch.float64))
        c = u * min(1.0, float(torch.tensor(max_norm)) / want)
        within(scale, torch.tensor([c], device="cuda", dtype=torch.float64), 5 * U * abs(c))
        again = plan.clip(max_norm, scale_of)
        assert torch.equal(again[0], norm) and torch.equal(again[1], scale)
        for g, out in zip(grads, clipped):
            product = g.double() * c
            within(out, product, (6 * U + ROUND[g.dtype] * 1.01) * product.abs() + TINY * 2.0 ** -7)


def test_norm_at_the_ends_of_the_range():
    """The squares of these are infinite or vanish in binary32."""
    for value, n in ((1e25, 1000), (3e38, 1), (1e-30, 5000), (1e-38, 100)):
        g = torch.full((n,), value, device="cuda")
        want, _ = exact_norm([g])
        within(solo.SoloGradNorm([g]).norm()[0], torch.tensor([want], dtype=torch.float64, device="cuda"), 2 * U * want)
    norm, scale, _ = solo.SoloGradNorm([torch.full((1000,), 3e38, device="cuda")]).norm(1.0)
    assert norm.item() == math.inf and scale.item() == 0.0


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_that_are_not_finite(bad, dtype):
    """The scale is 0, and so is every clipped gradient."""
    grads = [randn(20_000, dtype, 1), randn(33, dtype, 2)]
    grads[0][17_001] = bad
    clipped = [torch.full_like(g, 7.0) for g in grads]
    norm, scale, each = solo.SoloGradNorm(grads, clipped).clip(1.0)
    assert not math.isfinite(norm.item()) and scale.item() == 0.0
    assert not math.isfinite(each[0].item()) and math.isfinite(each[1].item())
    assert all(int(c.count_nonzero()) == 0 for c in clipped)


def test_clip_in_place():
    grads = [randn(30_001, torch.float32, 1), randn(5, torch.bfloat16, 2)]
    before = [g.clone() for g in grads]
    plan = solo.SoloGradNorm(grads, grads)
    want, _ = exact_norm(grads)
    plan.clip(2 * want)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))       # nothing to clip
    _, scale, _ = plan.clip(want / 4)
    for g, b in zip(grads, before):
        assert torch.equal(g, (b.float() * scale).to(b.dtype))
    within(plan.norm()[0], torch.tensor([want / 4], device="cuda"), 2.0 ** -8 * want)


def test_nothing_but_empty_tensors():
    plan = solo.SoloGradNorm([torch.empty(0, device="cuda")], [torch.empty(0, device="cuda")])
    norm, scale, each = plan.clip(1.0)
    assert norm.item() == 0.0 and scale.item() == 1.0 and each.tolist() == [0.0]


def test_norm_of_more_elements_than_32_bits_count():
    n = (1 << 32) + 5
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[(1 << 32) - 1], g[-1] = 3.0, 4.0, 12.0
    plan = solo.SoloGradNorm([g, g[1:9]], [g, None])
    norm, _, each = plan.clip(6.5)
    assert norm.item() == 13.0 and each.tolist() == [13.0, 0.0]
    assert g[0].item() == 1.5 and g[(1 << 32) - 1].item() == 2.0 and g[-1].item() == 6.0
    assert int(g.count_nonzero()) == 3


def test_the_scale_feeds_the_step():
    """grad_scale on the GPU, into the step, is the step of clipped gradients."""
    n = 10_000
    cfg = solo.make_config(4, 4, 128, solo.SOLO_GRAD_FP32)
    g = randn(n, torch.float32, 3)
    scaled = torch.empty_like(g)
    results = []
    for clip in (False, True):
        p, state, plan = randn(n, torch.float32, 4), solo.SoloState(n, cfg), solo.SoloGradNorm([g], [scaled])
        if clip:
            plan.clip(1.0)
            state.step(p, scaled, 1)
        else:
            state.step(p, g, 1, grad_scale=plan.norm(1.0)[1])
        results.append((p, *state.buffers()))
    assert all(torch.equal(a, b) for a, b in zip(*results))


# ---- embedding -------------------------------------------------------------------------------

def tokens_of(kind, n, vocab, seed, dtype=torch.int64):
    gen = generator(seed)
    if kind == "same":
        ids = torch.full((n,), vocab // 2, device="cuda")
    elif kind == "few":
        ids = torch.randint(0, max(1, vocab // 20), (n,), generator=gen, device="cuda")
    else:
        ids = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    if kind == "padded":
        ids[torch.rand(n, generator=gen, device="cuda") < 0.5] = -1
        ids[torch.rand(n, generator=gen, device="cuda") < 0.1] = vocab
        ids[torch.rand(n, generator=gen, device="cuda") < 0.1] = -(1 << 31)
    return ids.to(dtype)


def strided(rows, cols, dtype, seed, extra, scale=1.0):
    return randn((rows, cols + extra), dtype, seed, scale)[:, extra // 2:extra // 2 + cols]


def exact_lookup(table, ids, scale):
    known = (ids >= 0) & (ids < table.shape[0])
    return torch.where(known[:, None], table.double()[torch.where(known, ids, 0).long()] * scale, 0.0)


def exact_gradient(rows, ids, vocab, scale):
    """The gradient and the sum of its parts' absolute values, and the number of parts."""
    known = (ids >= 0) & (ids < vocab)
    ids, rows = ids[known].long().cpu(), rows[known].double().cpu() * scale
    zero = torch.zeros((vocab, rows.shape[1]), dtype=torch.float64)
    count = torch.zeros(vocab, dtype=torch.float64).index_add_(0, ids, torch.ones(len(ids), dtype=torch.float64))
    return [x.cuda() for x in (zero.clone().index_add_(0, ids, rows), zero.index_add_(0, ids, rows.abs()), count[:, None])]


@pytest.mark.parametrize("ids_dtype", [torch.int64, torch.int32])
@pytest.mark.parametrize("n,vocab,dim,extra", [(1, 1, 1, 0), (3, 50, 7, 0), (17, 100, 64, 3), (1000, 33, 100, 8), (257, 1000, 2056, 0), (5, 9, 4099, 1)])
@pytest.mark.parametrize("out_dtype", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_lookup(dtype, out_dtype, n, vocab, dim, extra, ids_dtype):
    table, ids = strided(vocab, dim, dtype, 1, extra), tokens_of("padded", n, vocab, 2, ids_dtype)
    whole = torch.full((n, dim + extra), 7.0, dtype=out_dtype, device="cuda")
    plan = solo.SoloEmbedding(vocab, dim, n + 5, scale=1.7)
    out = plan.lookup(table, ids, whole[:, extra:])
    want = exact_lookup(table, ids, float(torch.tensor(1.7)))
    within(out, want, (U + ROUND[out_dtype]) * 1.01 * want.abs())      # the product, then the output's type
    assert bool((whole[:, :extra] == 7.0).all())           # nothing beside the rows
    assert bool((out[(ids < 0) | (ids >= vocab)] == 0).all())


GRADS = [(1, 1, 1, 0, "any"), (3, 50, 7, 0, "any"), (31, 5, 8, 0, "few"), (32, 40, 24, 0, "same"), (33, 40, 24, 1, "same"), (64, 70, 65, 0, "same"),
         (500, 40, 9, 0, "padded"), (1000, 3, 64, 2, "any"), (1025, 2000, 130, 0, "few"), (3000, 700, 515, 5, "few"),
         (4097, 17, 40, 0, "padded"), (5000, 1, 16, 0, "same"), (2049, 9000, 33, 0, "any"), (700, 600, 1000, 8, "few"), (96, 3000, 768, 0, "any"),
         (256, 300, 64, 0, "few"), (257, 300, 64, 0, "few"), (2000, 600, 4099, 0, "few"), (3000, 40, 129, 0, "few"), (3000, 40, 255, 1, "same"), (3000, 40, 257, 0, "few"), (900, 30, 515, 0, "same"), (40_000, 50, 8, 0, "few"), (300_000, 70_000, 1, 0, "any")]


@pytest.mark.parametrize("ids_dtype", [torch.int64, torch.int32])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,vocab,dim,extra,kind", GRADS)
@pytest.mark.parametrize("dtype,out_dtype", [(a, b) for a in TYPES for b in TYPES])
def test_embedding_gradient(dtype, out_dtype, n, vocab, dim, extra, kind, accumulate, ids_dtype):
    rows, ids = strided(n, dim, dtype, 1, extra), tokens_of(kind, n, vocab, 2, ids_dtype)
    whole = randn((vocab, dim + extra), out_dtype, 3)
    before = whole.double()
    plan = solo.SoloEmbedding(vocab, dim, n + 9, scale=0.3)
    plan.grad(rows, ids, whole[:, extra:], accumulate=accumulate)
    want, size, count = exact_gradient(rows, ids, vocab, float(torch.tensor(0.3)))
    add = before[:, extra:] if accumulate else torch.zeros_like(want)
    # at most one rounding for every row that is added, one for the factor, one for the old value, one for the type
    bound = (count + 3) * U * 1.01 * (size + add.abs()) + ROUND[out_dtype] * 1.01 * (want + add).abs()
    within(whole[:, extra:], want + add, torch.where(count > 0, bound, 0.0))
    assert torch.equal(whole[:, :extra].double(), before[:, :extra])
    if not accumulate:
        assert bool((whole[:, extra:][count[:, 0] == 0] == 0).all())


def test_embedding_gradient_is_the_lookups_adjoint():
    """<lookup(E), dy> = <E, gradient(dy)>, and a step along one entry changes the product by the gradient's entry."""
    n, vocab, dim = 300, 40, 24
    ids, plan = tokens_of("padded", n, vocab, 1), solo.SoloEmbedding(vocab, dim, n, scale=0.5)
    table, dy = randn((vocab, dim), torch.float32, 2), randn((n, dim), torch.float32, 3)
    loss = lambda t: float((plan.lookup(t, ids, torch.empty_like(dy)).double() * dy.double()).sum())     # noqa: E731
    grad = plan.grad(dy, ids, torch.empty_like(table))
    dot, size = float((table.double() * grad.double()).sum()), float((table.double() * grad.double()).abs().sum())
    assert abs(loss(table) - dot) <= n * U * (size + n * dim)
    for v, c in ((0, 0), (39, 23), (7, 5)):
        there = table.clone()
        there[v, c] += 1.0
        step = float(there[v, c].double() - table[v, c].double())
        assert abs((loss(there) - loss(table)) - step * float(grad[v, c])) <= 1e-4       # sums of 7200 values near 1, u each


def test_embedding_gradient_without_tokens():
    plan = solo.SoloEmbedding(10, 20, 5)
    out = torch.full((10, 20), 7.0, device="cuda")
    none, rows = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty((0, 20), device="cuda")
    plan.grad(rows, none, out, accumulate=True)
    assert bool((out == 7).all())
    plan.grad(rows, none, out)
    assert bool((out == 0).all())
    assert plan.lookup(out, none, rows) is rows
    padding = torch.full((5,), -1, device="cuda")
    plan.grad(torch.full((5, 20), math.nan, device="cuda"), padding, out.fill_(7.0))
    assert bool((out == 0).all())


def test_embedding_gradient_is_the_same_on_every_call():
    n, vocab, dim = 20_000, 300, 520
    ids, dy = tokens_of("few", n, vocab, 1), randn((n, dim), torch.bfloat16, 2)
    plan = solo.SoloEmbedding(vocab, dim, n)
    first = plan.grad(dy, ids, torch.empty((vocab, dim), device="cuda")).clone()
    for _ in range(3):
        assert torch.equal(first, plan.grad(dy, ids, torch.empty((vocab, dim), device="cuda")))


def test_embedding_rows_that_lie_more_than_32_bits_apart():
    stride = (1 << 31) - 8
    buffer = torch.zeros(2 * stride + 16, dtype=torch.bfloat16, device="cuda")
    table = buffer.as_strided((3, 16), (stride, 1))
    table[2] = torch.arange(16, device="cuda")
    ids = torch.tensor([2, 0, 2], device="cuda")
    plan = solo.SoloEmbedding(3, 16, 3)
    out = plan.lookup(table, ids, torch.empty((3, 16), device="cuda"))
    assert out[0].tolist() == list(range(16)) == out[2].tolist() and not out[1].any()
    plan.grad(out, ids, table)
    assert table[2].tolist() == [2.0 * x for x in range(16)] and not table[:2].any()
    assert int(buffer.count_nonzero()) == 15
    rows = buffer.as_strided((3, 16), (stride, 1))
    assert plan.lookup(out, torch.tensor([1, 1, 0], device="cuda"), rows)[2].tolist() == list(range(16))


# ---- log probabilities -----------------------------------------------------------------------

def exact_rows(x, t, scale, a, b):
    """Log probability, entropy, rank, order of the columns, log p and the gradient, in 64 bits on the CPU."""
    x, t = x.double().cpu(), t.long().cpu()
    cols = x.shape[1]
    row = (t >= 0) & (t < cols)
    x = torch.where(row[:, None], x, 0.0)                  # (rows without a target may hold anything)
    z = x * scale
    m = z.amax(1, keepdim=True)
    empty = m[:, 0] == -math.inf
    d = torch.where(empty[:, None], -math.inf, z - torch.where(empty[:, None], 0.0, m))
    e = d.exp()
    s = e.sum(1, keepdim=True)
    logp = torch.where(empty[:, None], -math.inf, d - s.log())
    p = torch.where(empty[:, None], 0.0, logp.exp())
    plogp = torch.where(p > 0, p * logp, 0.0)
    entropy = torch.where(empty, 0.0, -plogp.sum(1))
    at = torch.where(row, t, 0)[:, None]
    logprob = logp.gather(1, at)[:, 0]
    rank = (x > x.gather(1, at)).sum(1)
    order = torch.argsort(x, dim=1, descending=True, stable=True)
    a, b = a.double().cpu()[:, None], b.double().cpu()[:, None]
    grad = -a * p - b * (plogp + p * entropy[:, None])
    grad.scatter_add_(1, at, torch.where(empty[:, None], 0.0, a))
    grad = torch.where(row[:, None], grad * scale, 0.0)
    reach = torch.where(e > 0, -d, 0.0).clamp(max=100).amax(1)            # how far the logits that count lie below the largest
    return [v.cuda() for v in (torch.where(row, logprob, 0.0), torch.where(row, entropy, 0.0), torch.where(row, rank, -1), order, logp, grad, row, p, reach)]


def check_rows(x, t, scale, top, seed=5, in_place=True):
    """Every result of the three calls against 64 bits."""
    rows, cols = x.shape
    scale = float(torch.tensor(scale))
    a, b = randn(rows, torch.float32, seed), randn(rows, torch.float32, seed + 1)
    logprob, entropy, rank, order, logp, grad, row, p, reach = exact_rows(x, t, scale, a, b)
    plan = solo.SoloLogprob(rows, cols, top=top, rank=True, scale=scale)
    got = [v.clone() for v in plan.forward(x, t)]
    # a thread adds up to cols / 256 + 8 values, 10 steps join the threads: eps.  A difference, its factor and the
    # exponential are 4 u of the distance (in units of ln 2 up to 1.5 of it) and of the value.
    eps = (cols / 256 + 32) * U
    off = 8 * U * (1 + reach) + eps
    within(got[0], logprob, off + 4 * U * logprob.abs().nan_to_num(posinf=0))
    off_entropy = (8 * U + eps) * (2 + 2 * reach + entropy)
    within(got[1], entropy, off_entropy)
    assert torch.equal(got[2], rank.int())
    if top:
        k = min(top, cols)
        want = torch.where(row[:, None], order[:, :k], -1)
        assert torch.equal(got[4][:, :k], want.int())
        value = torch.where(row[:, None], logp.gather(1, order[:, :k]), -math.inf)
        within(got[3][:, :k], value, off[:, None] + 4 * U * value.abs().nan_to_num(posinf=0))
        assert bool((got[4][:, k:] == -1).all()) and bool((got[3][:, k:] == -math.inf).all())
    # the gradient: relative errors of p, and the distance's error where it stands as a factor
    a, b, row_off = a.double().abs()[:, None], b.double().abs()[:, None], off[:, None]
    inner = torch.where(p > 0, logp, 0.0).abs() + entropy[:, None].abs()
    bound = scale * (p * (a * 4 * row_off + b * (inner * 4 * row_off + 2 * row_off + off_entropy[:, None] + 8 * U * inner)) + a * 4 * U * (p + (p > 0.25)))
    bound = bound + ROUND[x.dtype] * 1.01 * grad.abs() + 8 * U * a * scale * (torch.arange(cols, device="cuda") == t[:, None]) + TINY
    bound = torch.where(row[:, None], bound, 0.0)
    one, two = torch.empty_like(x), torch.empty_like(x)
    a, b = randn(rows, torch.float32, seed), randn(rows, torch.float32, seed + 1)
    within(plan.grad(x, t, a, b, two), grad, bound)
    lp, h, _ = plan.forward_grad(x, t, a, b, one)
    within(lp, logprob, off + 4 * U * logprob.abs().nan_to_num(posinf=0))
    within(h, entropy, off_entropy)
    within(one, grad, bound)
    if in_place:
        plan.forward(x, t)
        work = x.clone()
        assert torch.equal(plan.grad(work, t, a, b, work), two)
        work = x.clone()
        assert torch.equal(plan.forward_grad(work, t, a, b, work)[2], one)


SHAPES = [(1, 1), (1, 7), (3, 8), (2, 9), (5, 64), (4, 1000), (2, 2048 * 8), (3, 8 * 1024 + 3), (600, 5), (513, 300), (600, 2049), (2, 50257)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("scale,top", [(1.0, 5), (0.7, 0), (2.5, 32)])
def test_rows(rows, cols, dtype, scale, top):
    x = randn((rows, cols), dtype, rows + cols, 3.0)
    check_rows(x, torch.randint(0, cols, (rows,), generator=generator(9), device="cuda"), scale, top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [7, 700])
def test_rows_with_strides_masks_and_padding(rows, dtype):
    """Rows that begin anywhere, masked columns in several ways, rows without a target that hold NaN."""
    cols = 1003
    buffer = randn((rows, cols + 6), dtype, 1, 3.0)
    x = buffer[:, 3:3 + cols]
    lowest = torch.finfo(dtype).min
    x[0] = -math.inf                                       # nothing is left
    x[1] = lowest                                          # everything is as unlikely as can be: all alike
    x[2, 1:] = -math.inf                                   # one is left
    x[3, ::2] = lowest
    x[4, :500] = -math.inf
    x[5] = 0.0
    x[5, ::3] = -0.0
    t = torch.randint(0, cols, (rows,), generator=generator(9), device="cuda", dtype=torch.int32)
    t[2], t[6] = 0, -100
    x[6] = math.nan
    if rows > 7:
        t[650], t[660], t[670] = cols, -1, 2 ** 31 - 1
    keep = buffer.clone()
    check_rows(x, t, 1.3, 20, in_place=False)
    assert torch.equal(buffer.nan_to_num(nan=5.0), keep.nan_to_num(nan=5.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [3, 520])
def test_alternatives_among_equal_logits(rows, dtype):
    """Ties go to the lower column; large logits that all belong to a few threads' share of the row."""
    cols = 20_000
    x = torch.zeros((rows, cols), dtype=dtype, device="cuda")
    x[1] = torch.randint(0, 3, (cols,), generator=generator(1), device="cuda").to(dtype)
    share = torch.arange(cols, device="cuda") // 8 % 256 < 2
    x[2] = torch.where(share, 5.0 + torch.randint(0, 9, (cols,), generator=generator(2), device="cuda"), -torch.rand(cols, generator=generator(3), device="cuda")).to(dtype)
    check_rows(x, torch.full((rows,), 11, device="cuda"), 1.0, 32)


@pytest.mark.parametrize("rows", [2, 600])
def test_many_candidates(rows):
    """More elements above the last alternative's thread than are collected at once."""
    cols = 8 * 256 * 40
    x = torch.zeros((rows, cols), dtype=torch.float32, device="cuda")
    column = torch.arange(cols, device="cuda")
    hot = (column // 8 % 256 < 40)
    x[0] = torch.where(hot, 10.0 + (column * 7919 % 1000) * 1e-3, 0.0)
    x[1] = torch.where(column // 8 % 1024 < 40, 10.0 + column * 1e-5, 0.0)
    check_rows(x, torch.zeros(rows, dtype=torch.int64, device="cuda"), 1.0, 32)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("rows", [2, 600])
def test_logits_that_are_no_numbers(rows, bad):
    """NaN where the row holds one; whole alternatives of columns that exist; other rows as if it were not there."""
    cols = 5000
    x = randn((rows, cols), torch.float32, 1)
    clean = x.clone()
    x[1, 4321] = bad
    t = torch.full((rows,), 3, device="cuda")
    plan = solo.SoloLogprob(rows, cols, top=7)
    want = [v.clone() for v in plan.forward(clean, t)]
    got = plan.forward(x, t)
    others = torch.arange(rows, device="cuda") != 1
    assert all(torch.equal(g[others], w[others]) for g, w in zip(got, want))
    assert got[0][1].isnan() and got[1][1].isnan()
    assert bool(((got[3] >= 0) & (got[3] < cols)).all())
    a = torch.ones(rows, device="cuda")
    grad = plan.grad(x, t, a, a, torch.empty_like(x))
    assert bool(grad[1].isnan().any()) and bool(grad[0].isfinite().all())


def test_extreme_logits():
    cols = 300
    x = randn((4, cols), torch.float32, 1)
    x[0] *= 1e30                                           # the largest has all of it
    x[1] *= 1e-30
    x[2] += 1e4
    x[3, 0] = 3e38
    t = x.argmax(1)
    check_rows(x, t, 1.0, 3)


def test_rows_without_targets():
    x = randn((30, 700), torch.bfloat16, 1)
    plan = solo.SoloLogprob(40, 700, top=3, rank=True)
    t = torch.zeros(30, dtype=torch.int64, device="cuda")
    want = [v.clone() for v in plan.forward(x, t)]
    logprob, entropy, rank, value, token = plan.forward(x, None)
    assert logprob is None and rank is None
    assert torch.equal(entropy, want[1]) and torch.equal(value, want[3]) and torch.equal(token, want[4])
    b = torch.ones(30, device="cuda")
    with_targets = plan.grad(x, t, None, b, torch.empty_like(x))
    assert torch.equal(with_targets, plan.grad(x, None, None, b, torch.empty_like(x)))
    one = plan.forward_grad(x, None, None, b, torch.empty_like(x))[2]
    within(one, with_targets, 2.0 ** -7 * with_targets.double().abs() + 1e-6)     # (one place of bfloat16; values near 0 carry the sums' error)
    assert float(with_targets.float().abs().sum()) > 0


def test_empty_shapes():
    plan = solo.SoloLogprob(4, 0, top=2, rank=True)
    x = torch.empty((4, 0), device="cuda")
    logprob, entropy, rank, value, token = plan.forward(x, torch.zeros(4, dtype=torch.int64, device="cuda"))
    assert logprob.tolist() == [0.0] * 4 and entropy.tolist() == [0.0] * 4 and rank.tolist() == [-1] * 4
    assert bool((value == -math.inf).all()) and bool((token == -1).all())
    plan = solo.SoloLogprob(4, 9)
    none = torch.empty((0, 9), device="cuda")
    assert plan.forward(none, torch.empty(0, dtype=torch.int64, device="cuda"))[0].numel() == 0


def test_gradient_against_differences():
    """Central differences of the forward call along random directions v, |v| <= 1: the third derivative of either result along v is
    below 60 (the third cumulant of a variable in [-1, 1], and its product with log p + entropy, |.| <= 12); h = 2^-5 makes that
    60 h^2 / 6, and the results' error, 2e-6, is divided by h."""
    rows, cols, h = 6, 40, 2.0 ** -5
    x, t = randn((rows, cols), torch.float32, 1, 2.0), torch.arange(rows, device="cuda")
    a, b = randn(rows, torch.float32, 2), randn(rows, torch.float32, 3)
    plan = solo.SoloLogprob(rows, cols)

    def loss(y):
        lp, entropy = plan.forward(y, t)
        return a.double() * lp.double() + b.double() * entropy.double()

    plan.forward(x, t)
    grad = plan.grad(x, t, a, b, torch.empty_like(x)).double()
    for seed in range(4, 10):
        v = torch.rand((rows, cols), generator=generator(seed), device="cuda") * 2 - 1
        up, down = x + h * v, x - h * v
        difference = (loss(up) - loss(down)) / 2 / h
        along = (grad * (up.double() - down.double()) / 2 / h).sum(1)
        within(difference, along, (60 * h * h / 6 + 2e-6 / h) * (a.abs() + b.abs()))


def test_logits_that_lie_more_than_32_bits_apart():
    stride, cols = (1 << 31) + 8, 100
    buffer = torch.zeros(2 * stride + cols, dtype=torch.bfloat16, device="cuda")
    x = buffer.as_strided((3, cols), (stride, 1))
    x.copy_(randn((3, cols), torch.bfloat16, 1))
    t = torch.tensor([5, 6, 7], device="cuda")
    plan, near = solo.SoloLogprob(3, cols, top=4), x.contiguous()
    want = [v.clone() for v in plan.forward(near, t)]
    assert all(torch.equal(g, w) for g, w in zip(plan.forward(x, t), want))
    a = torch.ones(3, device="cuda")
    grad = plan.grad(near, t, a, None, torch.empty_like(near))
    assert torch.equal(plan.grad(x, t, a, None, x), grad)


# ---- streams and graphs ----------------------------------------------------------------------

def everything():
    """One call of each operator on buffers of its own: (call, outputs)."""
    n, vocab, dim = 3000, 500, 264
    table, ids, dy = randn((vocab, dim), torch.bfloat16, 1), tokens_of("few", n, vocab, 2), randn((n, dim), torch.bfloat16, 3)
    rows, grad_table = torch.empty((n, dim), device="cuda"), torch.empty((vocab, dim), device="cuda")
    embed = solo.SoloEmbedding(vocab, dim, n)
    embed.grad(dy, ids, grad_table)                        # (the workspace)
    few_ids, few_table = tokens_of("few", 50, vocab, 4), torch.empty((vocab, dim), device="cuda")
    x, t = randn((600, 3001), torch.bfloat16, 5), torch.randint(0, 3001, (600,), generator=generator(6), device="cuda")
    a = randn(600, torch.float32, 7)
    logprob, other, dx, dx_one = solo.SoloLogprob(600, 3001, top=6, rank=True), solo.SoloLogprob(600, 3001), torch.empty_like(x), torch.empty_like(x)
    few = solo.SoloLogprob(2, 3001, top=6)
    grads = [dx.view(-1), grad_table.view(-1)]
    clipped = [torch.empty_like(g) for g in grads]
    norm = solo.SoloGradNorm(grads, clipped)

    def call(stream=None):
        embed.lookup(table, ids, rows, stream=stream)
        embed.grad(dy, ids, grad_table, stream=stream)
        embed.grad(dy[:50], few_ids, few_table, stream=stream)
        logprob.forward(x, t, stream=stream)
        logprob.grad(x, t, a, a, dx, stream=stream)
        other.forward_grad(x, t, a, a, dx_one, stream=stream)
        few.forward(x[:2], t[:2], stream=stream)
        norm.clip(1.0, stream=stream)

    outs = [rows, grad_table, few_table, logprob.logprob, logprob.entropy, logprob.rank, logprob.top_logprob, logprob.top_token, dx, dx_one,
            few.top_token, few.logprob, *norm.results, *clipped]
    return call, outs, (x, dy)


def test_another_stream():
    call, outs, _ = everything()
    call()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    for o in outs:
        o.zero_()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    call(stream)
    stream.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_graph():
    """Captured once, replayed with other inputs in the same buffers, between eager work."""
    call, outs, inputs = everything()
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(4):
        for x in inputs:
            x.copy_(randn(x.shape, x.dtype, 100 + seed))
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, got))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,top", [(1, 16384, 5), (128, 16389, 3), (7, 20_001, 32), (1, 300_003, 20), (2, 400_001, 0), (5, 65_537, 1)])
def test_few_long_rows(rows, cols, top, dtype):
    x = randn((rows, cols + 1), dtype, 1, 3.0)[:, 1:]
    t = torch.randint(0, cols, (rows,), generator=generator(9), device="cuda")
    if rows > 4:
        x[1] = -math.inf
        x[2, : cols - 5] = -math.inf
        x[3] = torch.finfo(dtype).min
        t[4] = -100
        x[4] = math.nan
    check_rows(x, t, 0.9, top, in_place=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("last", [2048, 8192, 16384, 32768, 65536])
@pytest.mark.parametrize("more", [0, 1, 3, 4, 5, 7, 8])
def test_rows_that_just_stay_in_registers_and_just_do_not(last, more, dtype):
    cols = last + more
    x = randn((3, cols), dtype, more, 3.0)
    x[:, last - 9:] += 9.0                                 # (what lies behind the line counts)
    check_rows(x, torch.tensor([cols - 1, 0, last - 1], device="cuda"), 1.0, 2)

