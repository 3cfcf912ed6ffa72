"""What the operators around the step refuse, and their host-side helpers (no GPU: every call returns before a launch)."""
import ctypes as C
import math

import pytest
import torch

from paper_2505_00347_amd import solo
from test_binding_loading import fresh_binding

BAD = solo.SOLO_E_INVALID


def norm_args(**changes):
    args = dict(table_device=16, count=1, units=1, unscale=None, max_norm=1.0, norm=16, grad_scale=16, tensor_norm=None, workspace=16)
    args.update(changes)
    return list(args.values())


@pytest.mark.parametrize("changes", [dict(max_norm=-1.0), dict(max_norm=math.nan), dict(count=0), dict(table_device=None), dict(table_device=8),
                                     dict(norm=None), dict(norm=2), dict(grad_scale=None), dict(tensor_norm=2), dict(unscale=2),
                                     dict(workspace=None), dict(workspace=8)])
def test_norm_refusals(changes):
    for call in (solo.solo_grad_norm, solo.solo_grad_clip):
        assert call(*norm_args(**changes), stream=0, check=False) == BAD
        with pytest.raises(solo.SoloError):
            call(*norm_args(**changes), stream=0)
    assert solo.solo_grad_norm(*norm_args(units=1 << 24), stream=0, check=False) == solo.SOLO_E_UNSUPPORTED


def test_norm_table():
    grads = (solo.solo_grad * 3)(solo.solo_grad(32, None, 40_000, solo.SOLO_FP32, 0), solo.solo_grad(None, None, 0, 1, 0),
                                 solo.solo_grad(34, 66, 5, solo.SOLO_BF16, 0))
    units = solo.solo_norm_units(grads, 3)
    assert units == 4
    size = solo.solo_norm_table_bytes(3, units)
    assert size == 3 * 48 + 4 * 4
    host = (C.c_uint32 * (size // 4))()
    assert solo.solo_norm_table_build(grads, 3, C.addressof(host), size) == solo.SOLO_OK
    assert list(host)[36:] == [0, 0, 0, 2]
    assert solo.solo_norm_table_build(grads, 3, C.addressof(host), size - 1, check=False) == BAD
    assert solo.solo_norm_table_build(grads, 3, None, size, check=False) == BAD
    assert solo.solo_norm_table_build(grads, 0, C.addressof(host), size, check=False) == BAD
    for change in (dict(grad=33), dict(clipped=67), dict(dtype=2), dict(reserved=1), dict(grad=None)):
        bad = (solo.solo_grad * 1)(grads[2])
        for name, value in change.items():
            setattr(bad[0], name, value)
        assert solo.solo_norm_table_build(bad, 1, C.addressof(host), size, check=False) == BAD, change
    bad[0] = solo.solo_grad(32, None, (1 << 40) + 1, 0, 0)
    assert solo.solo_norm_units(bad, 1) == 0
    assert solo.solo_norm_table_build(bad, 1, C.addressof(host), size, check=False) == solo.SOLO_E_UNSUPPORTED
    # a large set has units of more elements, about 2^16 of them
    large = (solo.solo_grad * 2)(solo.solo_grad(32, None, 6_738_415_616, 1, 0), solo.solo_grad(32, None, 1, 1, 0))
    assert 1 << 14 <= solo.solo_norm_units(large, 2) <= 1 << 17


def shape(**changes):
    s = solo.solo_embedding_shape(10, 8, 4, 8, 8, 0, 1, 64, 0, 1.0, 0)
    for name, value in changes.items():
        setattr(s, name, value)
    return s


SHAPE_CHANGES = [dict(table_dtype=2), dict(rows_dtype=7), dict(token_bits=16), dict(flags=2), dict(scale=math.inf), dict(scale=math.nan),
                 dict(reserved=1), dict(table_stride=7), dict(rows_stride=7)]
TOO_LARGE = [dict(vocab=1 << 31), dict(tokens=1 << 28), dict(dim=1 << 24, table_stride=1 << 24, rows_stride=1 << 24), dict(table_stride=1 << 31)]


@pytest.mark.parametrize("changes", SHAPE_CHANGES)
def test_embedding_shapes_that_are_refused(changes):
    assert solo.solo_embedding(16, 16, 16, shape(**changes), stream=0, check=False) == BAD
    assert solo.solo_embedding_grad(16, 16, 16, 16, 1 << 40, shape(**changes), stream=0, check=False) == BAD
    assert solo.solo_embedding_workspace_bytes(shape(**changes)) == 0


@pytest.mark.parametrize("changes", TOO_LARGE)
def test_embedding_shapes_that_are_too_large(changes):
    assert solo.solo_embedding(16, 16, 16, shape(**changes), stream=0, check=False) == solo.SOLO_E_UNSUPPORTED
    assert solo.solo_embedding_grad(16, 16, 16, 16, 1 << 40, shape(**changes), stream=0, check=False) == solo.SOLO_E_UNSUPPORTED
    assert solo.solo_embedding_workspace_bytes(shape(**changes)) == 0


def test_embedding_pointers():
    s, enough = shape(), solo.solo_embedding_workspace_bytes(shape())
    assert enough > 0
    for args in ((None, 16, 16), (18, 16, 16), (16, None, 16), (16, 20, 16), (16, 16, None), (16, 16, 17)):
        assert solo.solo_embedding(*args, s, stream=0, check=False) == BAD, args
    for args in ((None, 16, 16, 16), (17, 16, 16, 16), (16, None, 16, 16), (16, 20, 16, 16), (16, 16, None, 16), (16, 16, 18, 16),
                 (16, 16, 16, None), (16, 16, 16, 8)):
        assert solo.solo_embedding_grad(*args, enough, s, stream=0, check=False) == BAD, args
    assert solo.solo_embedding_grad(16, 16, 16, 16, enough - 1, s, stream=0, check=False) == BAD
    assert solo.solo_embedding(16, 16, 16, shape(flags=1), stream=0, check=False) == BAD          # (a gradient's flag)
    assert solo.solo_embedding(None, None, None, shape(tokens=0), stream=0) == solo.SOLO_OK
    assert solo.solo_embedding(None, None, None, shape(dim=0), stream=0) == solo.SOLO_OK
    for nothing in (dict(vocab=0), dict(dim=0), dict(tokens=0, flags=1)):
        assert solo.solo_embedding_grad(None, None, None, None, 0, shape(**nothing), stream=0) == solo.SOLO_OK
    for wrong in (None, 16, solo.solo_logits()):
        with pytest.raises((C.ArgumentError, TypeError)):
            solo.solo_embedding(16, 16, 16, wrong, stream=0)


def test_embedding_workspace_grows_with_the_tokens():
    for vocab, dim in ((1, 1), (50257, 768), (32000, 4096), (300_000, 65)):
        sizes = [solo.solo_embedding_workspace_bytes(shape(vocab=vocab, dim=dim, table_stride=dim, rows_stride=dim, tokens=n))
                 for n in (0, 1, 31, 32, 33, 64, 100, 255, 256, 257, 1000, 1024, 4096, 4097, 8192, 10_000, 16384, 16385, 65536, 100_000, 131072, 10 ** 6)]
        assert sizes == sorted(sizes) and sizes[0] > 0


def logits(**changes):
    s = solo.solo_logits(4, 8, 8, 8, 0, 64, 2, 0, 1.0, 0)
    for name, value in changes.items():
        setattr(s, name, value)
    return s


@pytest.mark.parametrize("changes", [dict(dtype=2), dict(target_bits=8), dict(top=33), dict(reserved=1), dict(reserved2=1), dict(scale=0.0),
                                     dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(scale=3e38), dict(stride=7)])
def test_logits_that_are_refused(changes):
    s = logits(**changes)
    assert solo.solo_logprob(16, 16, 16, 16, 16, 16, 16, 16, s, stream=0, check=False) == BAD
    assert solo.solo_logprob_grad(16, 16, 16, 16, 16, 16, 16, s, stream=0, check=False) == BAD
    assert solo.solo_logprob_with_grad(16, 16, 16, 16, 16, 16, 16, s, stream=0, check=False) == BAD


def test_logits_pointers():
    s = logits()
    good = [16, 16, 16, 16, 16, 16, 16, 16]
    for at, bad in ((0, None), (0, 18), (1, None), (1, 20), (2, 18), (3, 18), (4, 18), (5, None), (5, 18), (6, None), (6, 18), (7, 18)):
        assert solo.solo_logprob(*good[:at], bad, *good[at + 1:], s, stream=0, check=False) == BAD, (at, bad)
    good = good[:7]
    for at, bad in ((0, None), (1, None), (1, 20), (2, None), (2, 18), (3, None), (3, 18), (4, 18), (5, 18), (6, None), (6, 18)):
        assert solo.solo_logprob_grad(*good[:at], bad, *good[at + 1:], s, stream=0, check=False) == BAD, (at, bad)
    assert solo.solo_logprob_grad(16, 16, 16, 16, None, None, 16, s, stream=0, check=False) == BAD
    assert solo.solo_logprob_grad(*good, logits(grad_stride=7), stream=0, check=False) == BAD
    for at, bad in ((0, None), (1, None), (1, 20), (2, 18), (3, 18), (4, 18), (5, 18), (6, None), (6, 18)):
        assert solo.solo_logprob_with_grad(*good[:at], bad, *good[at + 1:], s, stream=0, check=False) == BAD, (at, bad)
    assert solo.solo_logprob_with_grad(16, 16, None, None, 16, 16, 16, s, stream=0, check=False) == BAD
    assert solo.solo_logprob_with_grad(*good, logits(grad_stride=7), stream=0, check=False) == BAD
    nothing = [None] * 8
    assert solo.solo_logprob(*nothing, logits(rows=0), stream=0) == solo.SOLO_OK
    assert solo.solo_logprob_grad(*nothing[:7], logits(rows=0), stream=0) == solo.SOLO_OK
    assert solo.solo_logprob_with_grad(*nothing[:7], logits(rows=0), stream=0) == solo.SOLO_OK
    for large in (dict(cols=1 << 31, stride=1 << 31, grad_stride=1 << 31), dict(rows=1 << 40)):
        assert solo.solo_logprob(16, 16, 16, 16, 16, 16, 16, 16, logits(**large), stream=0, check=False) == solo.SOLO_E_UNSUPPORTED


@pytest.mark.parametrize("native", (True, False))
def test_both_ways_into_the_library_take_the_same_arguments(tmp_path, native):
    b = fresh_binding(tmp_path, native)

    class Tensor:
        def data_ptr(self):
            return 16

    assert b.solo_grad_norm(*norm_args(max_norm=-1), stream=0, check=False) == BAD                # (a whole number)
    assert b.solo_grad_norm(*norm_args(table_device=Tensor(), count=C.c_uint32(0)), stream=0, check=False) == BAD
    assert b.solo_grad_norm(*norm_args(max_norm=C.c_float(-1.0)), stream=0, check=False) == BAD
    s = b.solo_embedding_shape(10, 8, 0, 8, 8, 0, 1, 64, 0, 1.0, 0)
    assert b.solo_embedding(Tensor(), Tensor(), None, s, stream=0) == b.SOLO_OK
    s.tokens = 4
    assert b.solo_embedding_grad(Tensor(), Tensor(), Tensor(), Tensor(), 3, s, stream=0, check=False) == BAD
    x = b.solo_logits(0, 8, 8, 8, 0, 64, 2, 0, 1.0, 0)
    assert b.solo_logprob(Tensor(), *[None] * 7, x, stream=0) == b.SOLO_OK
    with pytest.raises((C.ArgumentError, TypeError)):
        b.solo_grad_norm(*norm_args(max_norm="1"), stream=0)
    with pytest.raises((C.ArgumentError, TypeError)):
        b.solo_grad_norm(*norm_args(count=1.5), stream=0)


def test_handles_refuse_what_does_not_fit():
    """The handles check shapes, types and strides of tensors before the library is called."""
    embed = solo.SoloEmbedding(10, 8, 4, device="cpu")
    table, ids, rows = torch.zeros(10, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4, 8)
    for t, i, r in ((table[:9], ids, rows), (table, ids, rows[:, :7]), (table, ids[:3], rows), (table.t().contiguous().t(), ids, rows),
                    (table, torch.zeros(5, dtype=torch.int64), torch.zeros(5, 8)), (table, torch.zeros(2, 2, dtype=torch.int64), rows),
                    (table, torch.zeros(8, dtype=torch.int64)[::2], rows), (table, ids, torch.zeros(1, 8).expand(4, 8))):
        with pytest.raises(ValueError):
            embed.lookup(t, i, r, stream=0)
        with pytest.raises(ValueError):
            embed.grad(r, i, t, stream=0)
    for t, i, r in ((table.double(), ids, rows), (table, ids.float(), rows), (table, ids, rows.half())):
        with pytest.raises(TypeError):
            embed.lookup(t, i, r, stream=0)
    with pytest.raises(solo.SoloError):
        solo.SoloEmbedding(10, 8, 1 << 28, device="cpu")
    plan = solo.SoloLogprob(4, 8, device="cpu")
    x, t, w = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    for args in ((torch.zeros(5, 8), torch.zeros(5, dtype=torch.int64)), (torch.zeros(4, 9), t), (x, t[:3]), (torch.zeros(8, 4).t(), t)):
        with pytest.raises(ValueError):
            plan.forward(*args, stream=0)
    for args in ((x, t, w[:3], None, x), (x, t, w, w.double(), x), (x, t, w, None, x[:3]), (x, t, torch.zeros(8)[::2], None, x)):
        with pytest.raises(ValueError):
            plan.grad(*args, stream=0)
        with pytest.raises(ValueError):
            plan.forward_grad(*args, stream=0)
    for args in ((x.half(), t), (x, t.short())):
        with pytest.raises(TypeError):
            plan.forward(*args, stream=0)
    with pytest.raises(TypeError):
        plan.grad(x, t, w, None, x.bfloat16(), stream=0)
    for top in (-1, 33):
        with pytest.raises(ValueError):
            solo.SoloLogprob(4, 8, top=top, device="cpu")
    g = torch.zeros(10)
    for grads, clipped in (([g[::2]], None), ([g], [g[:5]]), ([g], [g.bfloat16()]), ([g], [])):
        with pytest.raises(ValueError):
            solo.SoloGradNorm(grads, clipped, device="cpu")
    with pytest.raises(TypeError):
        solo.SoloGradNorm([g.double()], device="cpu")
    with pytest.raises(ValueError):
        solo.SoloGradNorm([g], device="cpu").clip(1.0, stream=0)
    with pytest.raises(TypeError):
        solo.SoloGradNorm([g], device="cpu").norm(1.0, unscale=torch.ones(1, dtype=torch.float64), stream=0)
