"""The operators around the step at sizes behind the lines of their dispatch, against plain implementations in 64 bits."""
import math

import pytest
import torch

from paper_2505_00347_amd import solo
from test_gpu_operators import ROUND, TINY, TYPES, U, exact_lookup, randn, strided, tokens_of, within

pytestmark = pytest.mark.gpu


def test_as_many_tokens_as_a_gradient_takes():
    """The parts of frequent tokens are more than one launch has workgroups for.  Whole numbers, whose sums are exact."""
    n, vocab = (1 << 28) - 1, 70_000
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, vocab, (n,), generator=gen, device="cuda", dtype=torch.int32)
    rows = torch.randint(-8, 9, (n, 1), generator=gen, device="cuda", dtype=torch.int8).bfloat16()
    out = solo.SoloEmbedding(vocab, 1, n).grad(rows, ids, torch.empty((vocab, 1), device="cuda"))
    want = torch.zeros(vocab, dtype=torch.float64, device="cuda")
    for at in range(0, n, 1 << 26):
        want.index_add_(0, ids[at:at + (1 << 26)], rows[at:at + (1 << 26), 0].double())
    assert torch.equal(out[:, 0].double(), want)


# The lines of the dispatch that go by bytes.  The kernels on the two sides are other ones, so that there are cases on both.
PAST_BYTES = 64 << 20               # looked-up rows, gradients of them
PAST_LOADS = 256 << 20              # logits
PAST_STORES = 32 << 20              # gradients of logits
LARGE_BYTES = 384 << 20             # gradients of a table of the norm


# ---- norm and clipping -----------------------------------------------------------------------

def norm_sizes(large, types):
    """Of three tensors: a few bytes more than the line, or a few less."""
    whole = LARGE_BYTES // max(t.itemsize for t in types)
    return [whole // 2 + 1, whole // 3 + 3, whole - (whole // 2 + 1) - (whole // 3 + 3) + (5 if large else -5)]


@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_norm_and_clip_around_the_line(dtype, large):
    sizes = norm_sizes(large, [dtype])
    grads = [randn(n + 3, dtype, n, 1e-3)[k + 1:][:n] for k, n in enumerate(sizes)]        # (begin anywhere)
    assert (sum(g.numel() * g.element_size() for g in grads) > LARGE_BYTES) == large
    squares = [sum(float(p.double().square().sum()) for p in g.split(1 << 26)) for g in grads]
    want, c = math.sqrt(sum(squares)), 0.25 / math.sqrt(sum(squares))
    clipped = [torch.full((n + 3,), 7.0, dtype=dtype, device="cuda")[3 - k:][:n] for k, n in enumerate(sizes)]
    norm, scale, each = solo.SoloGradNorm(grads, clipped).clip(0.25)
    # the bounds of the smaller sets: sums in binary64, one rounding to binary32; the factor's 5 u; product and type
    within(norm, torch.tensor([want], device="cuda"), 2 * U * want)
    each_want = torch.tensor(squares, dtype=torch.float64, device="cuda").sqrt()
    within(each, each_want, 2 * U * each_want)
    within(scale, torch.tensor([c], dtype=torch.float64, device="cuda"), 5 * U * c)
    plan = solo.SoloGradNorm(grads, grads)
    plan.clip(0.25)                                        # (in place)
    for k, (g, out) in enumerate(zip(grads, clipped)):
        assert torch.equal(g, out)
        original = randn(sizes[k] + 3, dtype, sizes[k], 1e-3)[k + 1:][:sizes[k]]
        for a, b in zip(original.split(1 << 26), out.split(1 << 26)):
            product = a.double() * c
            within(b, product, (6 * U + ROUND[dtype] * 1.01) * product.abs() + TINY * 2.0 ** -7)


# ---- embedding -------------------------------------------------------------------------------

def rows_around(past, dim, dtype):
    """Rows of `dim` columns that are just more bytes than the line, or just not."""
    return PAST_BYTES // (dim * dtype.itemsize) + (1 if past else 0)


DIMS = [1001, 100]                  # a wavefront for each row, and teams of fewer lanes


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("past", [False, True])
@pytest.mark.parametrize("ids_dtype", [torch.int64, torch.int32])
@pytest.mark.parametrize("dtype,out_dtype", [(a, b) for a in TYPES for b in TYPES])
def test_lookup_around_the_line(dtype, out_dtype, ids_dtype, past, dim):
    n, vocab = rows_around(past, dim, out_dtype), 3001
    table, ids = strided(vocab, dim, dtype, 1, 3), tokens_of("padded", n, vocab, 2, ids_dtype)
    whole = torch.full((n, dim + 1), 7.0, dtype=out_dtype, device="cuda")
    out = solo.SoloEmbedding(vocab, dim, n, scale=1.7).lookup(table, ids, whole[:, 1:])
    want = exact_lookup(table, ids, float(torch.tensor(1.7)))
    within(out, want, (U + ROUND[out_dtype]) * 1.01 * want.abs())      # the product, then the output's type
    assert bool((whole[:, 0] == 7.0).all())


def exact_gradient(rows, ids, vocab, scale):
    """The gradient, the sum of its parts' absolute values, and the number of parts."""
    known = (ids >= 0) & (ids < vocab)
    ids, rows = ids[known], rows[known].double() * scale
    zero = torch.zeros((vocab, rows.shape[1]), dtype=torch.float64, device="cuda")
    return zero.index_add(0, ids, rows), zero.index_add(0, ids, rows.abs()), torch.bincount(ids, minlength=vocab)[:, None]


@pytest.mark.parametrize("kind", ["few", "padded"])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("past", [False, True])
@pytest.mark.parametrize("dtype,out_dtype", [(a, b) for a in TYPES for b in TYPES])
def test_embedding_gradient_around_the_line(dtype, out_dtype, past, dim, kind):
    n, vocab = rows_around(past, dim, dtype), 2003
    rows, ids = strided(n, dim, dtype, 1, 3), tokens_of(kind, n, vocab, 2)
    plan, out = solo.SoloEmbedding(vocab, dim, n, scale=0.3), torch.empty((vocab, dim), dtype=out_dtype, device="cuda")
    want, size, count = exact_gradient(rows, ids, vocab, float(torch.tensor(0.3)))
    # a rounding for every row that is added, one for the factor, one for the type; then the same for the old value
    bound = (count + 3) * U * 1.01 * size + ROUND[out_dtype] * 1.01 * want.abs()
    within(plan.grad(rows, ids, out), want, bound)
    old = out.double()
    within(plan.grad(rows, ids, out, accumulate=True), want + old, torch.where(count > 0, bound + (3 * U + ROUND[out_dtype]) * 1.01 * (want.abs() + old.abs()), 0.0))


# ---- log probabilities -----------------------------------------------------------------------

# Columns for each number of threads that a row gets; rows for 2 MB, just behind the stores' line and just behind the loads' line.  Then few
# rows: with so many threads that they are read past the caches only where they are very long.
COLUMNS = [1003, 2003, 5003, 12_003, 20_003, 50_003, 70_003]
SIZES = [2 << 20, PAST_STORES, PAST_LOADS]
FEW_ROWS = [(5, 20_003), (100, 1_400_001)]


def logits_cases(dtype):
    return [(size // (cols * dtype.itemsize) + 1, cols) for size in SIZES for cols in COLUMNS] + FEW_ROWS


def exact(x, t, scale):
    """Log probability, entropy, rank, columns in order, ln p, rows with a target and p, in 64 bits; how far logits that count lie below the
    largest."""
    cols = x.shape[1]
    row = (t >= 0) & (t < cols)
    x = torch.where(row[:, None], x.double(), 0.0)
    largest = x.amax(1, keepdim=True)
    empty = largest == -math.inf
    d = torch.where(empty, -math.inf, (x - torch.where(empty, 0.0, largest)) * scale)
    e = d.exp()
    s = e.sum(1, keepdim=True)
    logp = torch.where(empty, -math.inf, d - s.log())
    p = torch.where(empty, 0.0, e / s)
    plogp = torch.where(p > 0, p * logp, 0.0)
    entropy = -plogp.sum(1, keepdim=True)
    at = torch.where(row, t, 0)[:, None]
    reach = torch.where(e > 0, -d, 0.0).clamp(max=100).amax(1)
    return (torch.where(row, logp.gather(1, at)[:, 0], 0.0), torch.where(row, entropy[:, 0], 0.0), torch.where(row, (x > x.gather(1, at)).sum(1), -1).int(),
            x.sort(dim=1, descending=True, stable=True).indices, logp, row, p, reach)


def exact_grad(p, logp, entropy, row, t, scale, a, b):
    grad = -a * p - b * torch.where(p > 0, p * (logp + entropy[:, None]), 0.0)
    some = p.amax(1, keepdim=True) > 0
    grad.scatter_add_(1, torch.where(row, t, 0)[:, None], torch.where(some, a, 0.0))
    return torch.where(row[:, None], grad * scale, 0.0)


@pytest.mark.parametrize("dtype,rows,cols", [(dtype, *case) for dtype in TYPES for case in logits_cases(dtype)])
def test_logits_around_the_lines(dtype, rows, cols):
    """Rows that begin anywhere, masked columns, rows with nothing and rows without a target, every call and every set of outputs."""
    scale, top = float(torch.tensor(1.3)), 20
    buffer = randn((rows, cols + 6), dtype, 1, 3.0)
    x = buffer[:, 3:3 + cols]
    x[:, ::7] = -math.inf
    x[1] = -math.inf
    x[2] = torch.finfo(dtype).min
    x[3], x[4] = math.nan, -math.inf
    x[4, 11] = 0.5
    t = torch.randint(0, cols, (rows,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    t[3] = -100
    a, b = randn(rows, torch.float32, 3), randn(rows, torch.float32, 4)
    results = {}
    for n, rank in ((top, True), (top, False), (0, True), (0, False)):
        plan = solo.SoloLogprob(rows, cols, top=n, rank=rank, scale=scale)
        results[n, rank] = [v.clone() for v in plan.forward(x, t)]
    grads = {}
    for weights in ((a, b), (a, None)):
        grads["two", weights[1] is b] = plan.grad(x, t, *weights, torch.full_like(buffer, 7.0)[:, 3:3 + cols])
        logprob, entropy, grads["one", weights[1] is b] = plan.forward_grad(x, t, *weights, torch.full_like(buffer, 7.0)[:, 3:3 + cols])
        results["one", weights[1] is b] = logprob.clone(), entropy.clone()
        for name in "two", "one":                          # in place
            work = buffer.clone()
            inside = work[:, 3:3 + cols]
            (plan.grad if name == "two" else plan.forward_grad)(inside, t, *weights, inside)
            assert torch.equal(inside, grads[name, weights[1] is b])
            assert torch.equal(work[:, :3], buffer[:, :3]) and torch.equal(work[:, 3 + cols:], buffer[:, 3 + cols:])
    step = max(1, 20_000_000 // cols)
    for i in range(0, rows, step):
        part = slice(i, i + step)
        a_, b_ = a[part].double()[:, None], b[part].double()[:, None]
        logprob, entropy, rank, order, logp, row, p, reach = exact(x[part], t[part], scale)
        # A thread adds cols / 64 values or fewer, some thirty steps join the threads: eps.  A difference, its factor and the exponential are
        # 4 u of the distance (in units of ln 2 up to 1.5 of it) and of the value.
        eps = (cols / 64 + 32) * U
        off = 8 * U * (1 + reach) + eps
        off_entropy = (8 * U + eps) * (2 + 2 * reach + entropy)
        for key, got in results.items():
            within(got[0][part], logprob, off + 4 * U * logprob.abs().nan_to_num(posinf=0))
            within(got[1][part], entropy, off_entropy)
            if key[1] is True and key[0] != "one":
                assert torch.equal(got[2][part], rank)
            if key[0] == top:
                assert torch.equal(got[-1][part], torch.where(row[:, None], order[:, :top], -1).int())
                value = torch.where(row[:, None], logp.gather(1, order[:, :top]), -math.inf)
                within(got[-2][part], value, off[:, None] + 4 * U * value.abs().nan_to_num(posinf=0))
        for (name, both), got in grads.items():
            grad = exact_grad(p, logp, entropy, row, t[part], scale, a_, b_ * both)
            size_a, size_b, row_off = a_.abs(), b_.abs() * both, off[:, None]
            inner = torch.where(p > 0, logp, 0.0).abs() + entropy[:, None].abs()
            bound = scale * (p * (size_a * 4 * row_off + size_b * (inner * 4 * row_off + 2 * row_off + off_entropy[:, None] + 8 * U * inner)) + size_a * 4 * U * (p + (p > 0.25)))
            bound = bound + ROUND[dtype] * 1.01 * grad.abs() + 8 * U * size_a * scale * (torch.arange(cols, device="cuda") == t[part][:, None]) + TINY
            within(got[part], grad, torch.where(row[:, None], bound, 0.0))
