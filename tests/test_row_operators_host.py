"""What layer norm, distillation and sampling refuse, and their handles (no GPU: every call returns before a launch)."""
import ctypes as C
import math

import pytest
import torch

from paper_2505_00347_amd import solo
from test_binding_loading import fresh_binding

BAD, TOO_LARGE = solo.SOLO_E_INVALID, solo.SOLO_E_UNSUPPORTED


def changed(struct, changes):
    for name, value in changes.items():
        setattr(struct, name, value)
    return struct


# ---- layer norm ------------------------------------------------------------------------------

def layer(**changes):
    return changed(solo.solo_layernorm_shape(4, 8, 8, 8, 8, 0, 1, 0, 0, 1e-5, 0), changes)


def layer_codes(s, room=1 << 50):
    return {solo.solo_layernorm(16, 16, 16, 16, 16, s, stream=0, check=False),
            solo.solo_layernorm_grad(16, 16, 16, 16, 16, 16, 16, 16, room, s, stream=0, check=False)}


@pytest.mark.parametrize("changes", [dict(x_dtype=2), dict(y_dtype=2), dict(weight_dtype=2), dict(flags=4), dict(reserved=1), dict(eps=0.0), dict(eps=-1e-5),
                                     dict(eps=math.inf), dict(eps=math.nan), dict(x_stride=7), dict(y_stride=7), dict(grad_stride=7)])
def test_layer_norm_shapes_that_are_refused(changes):
    assert layer_codes(layer(**changes)) == {BAD}
    assert solo.solo_layernorm_workspace_bytes(layer(**changes)) == 0


@pytest.mark.parametrize("changes", [dict(rows=1 << 31), dict(cols=1 << 24, x_stride=1 << 24, y_stride=1 << 24, grad_stride=1 << 24), dict(x_stride=1 << 31),
                                     dict(y_stride=1 << 31), dict(grad_stride=1 << 31)])
def test_layer_norm_shapes_that_are_too_large(changes):
    assert layer_codes(layer(**changes)) == {TOO_LARGE}
    assert solo.solo_layernorm_workspace_bytes(layer(**changes)) == 0


def test_layer_norm_pointers():
    s, enough = layer(), solo.solo_layernorm_workspace_bytes(layer())
    assert enough > 0
    good = [16, 16, 16, 16, 16]
    for at, bad in ((0, None), (0, 18), (1, 18), (2, 18), (3, None), (3, 17), (4, 18)):
        assert solo.solo_layernorm(*good[:at], bad, *good[at + 1:], s, stream=0, check=False) == BAD, (at, bad)
    good = [16] * 8
    for at, bad in ((0, None), (0, 17), (1, None), (1, 18), (2, 18), (3, None), (3, 18), (4, 18), (5, 18), (6, 18), (7, None), (7, 8)):
        assert solo.solo_layernorm_grad(*good[:at], bad, *good[at + 1:], enough, s, stream=0, check=False) == BAD, (at, bad)
    assert solo.solo_layernorm_grad(*good, enough - 1, s, stream=0, check=False) == BAD
    assert solo.solo_layernorm_grad(16, 16, 16, 16, None, None, None, 16, enough, s, stream=0, check=False) == BAD
    assert solo.solo_layernorm(*[16] * 5, layer(flags=2), stream=0, check=False) == BAD            # (a gradient's flag)
    for nothing in (dict(rows=0), dict(cols=0)):
        assert solo.solo_layernorm(*[None] * 5, layer(**nothing), stream=0) == solo.SOLO_OK
    assert solo.solo_layernorm_grad(*[None] * 8, 0, layer(cols=0), stream=0) == solo.SOLO_OK
    assert solo.solo_layernorm_grad(None, None, None, None, None, 16, None, None, 0, layer(rows=0, flags=2), stream=0) == solo.SOLO_OK
    for wrong in (None, 16, solo.solo_logits()):
        with pytest.raises((C.ArgumentError, TypeError)):
            solo.solo_layernorm(*[16] * 5, wrong, stream=0)


def test_layer_norm_workspace_grows_with_the_rows():
    for cols in (1, 64, 65, 300, 768, 1024, 2048, 4096, 5000, 16384, 16385, 300_000):
        strides = dict(cols=cols, x_stride=cols, y_stride=cols, grad_stride=cols)
        sizes = [solo.solo_layernorm_workspace_bytes(layer(rows=n, **strides)) for n in (0, 1, 2, 3, 31, 32, 33, 64, 100, 255, 256, 257, 1000, 1024, 5000, 10 ** 5, 10 ** 7)]
        assert sizes == sorted(sizes) and sizes[0] > 0


def test_layer_norm_handles_refuse_what_does_not_fit():
    plan = solo.SoloLayerNorm(4, 8, device="cpu")
    x, w = torch.zeros(4, 8), torch.zeros(8)
    for args in ((x[:, :7], w, w, x), (x, w[:7], w, x), (x, w, torch.zeros(16)[::2], x), (x, w, w, x[:3]), (torch.zeros(5, 8), w, w, torch.zeros(5, 8)),
                 (torch.zeros(8, 4).t(), w, w, x), (torch.zeros(32), w, w, x), (x, w, w, torch.zeros(1, 8).expand(4, 8)), (x, torch.zeros(1, 8), w, x)):
        with pytest.raises(ValueError):
            plan.forward(*args, stream=0)
    for args in ((x.double(), w, w, x), (x, w.half(), None, x), (x, w, w.bfloat16(), x), (x, w, w, x.half())):
        with pytest.raises(TypeError):
            plan.forward(*args, stream=0)
    with pytest.raises(ValueError, match="forward"):       # (nothing has been summed yet)
        plan.grad(x, x, w, x, w, w, stream=0)
    for args in ((x[:3], x, w, x, w, w), (x, x, w, x[:3], w, w), (x, x, w, x, w[:7], w), (x, x, w, x, w, torch.zeros(16)[::2])):
        with pytest.raises(ValueError):
            plan.grad(*args, stream=0)
    for args in ((x, x, w, x.bfloat16(), w, w), (x, x, w, x, w.bfloat16(), w), (x.half(), x, w, x, w, w)):
        with pytest.raises(TypeError):
            plan.grad(*args, stream=0)
    with pytest.raises(solo.SoloError):
        solo.SoloLayerNorm(4, 8, eps=0.0, device="cpu")
    with pytest.raises(solo.SoloError):
        solo.SoloLayerNorm(4, 1 << 24, device="cpu")


# ---- distillation ----------------------------------------------------------------------------

def distill(**changes):
    return changed(solo.solo_distill_shape(4, 8, 8, 8, 3, 3, 3, 0, 0, 64, 0, 0, 1.0, 1.0), changes)


def distill_codes(s):
    return {solo.solo_distill(16, 16, 16, 16, 16, s, stream=0, check=False), solo.solo_distill_grad(16, 16, 16, 16, 16, 16, s, stream=0, check=False),
            solo.solo_distill_with_grad(16, 16, 16, 16, 16, 16, s, stream=0, check=False)}


@pytest.mark.parametrize("changes", [dict(dtype=2), dict(value_dtype=2), dict(token_bits=16), dict(top=0), dict(top=129, value_stride=200, token_stride=200),
                                     dict(flags=2), dict(reserved=1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan),
                                     dict(scale=3e38), dict(teacher_scale=0.0), dict(teacher_scale=math.nan), dict(flags=1, teacher_scale=2.0),
                                     dict(stride=7), dict(value_stride=2), dict(token_stride=2)])
def test_distillation_shapes_that_are_refused(changes):
    assert distill_codes(distill(**changes)) == {BAD}


@pytest.mark.parametrize("changes", [dict(cols=1 << 29, stride=1 << 29, grad_stride=1 << 29), dict(rows=1 << 35), dict(stride=1 << 40), dict(grad_stride=1 << 40),
                                     dict(value_stride=1 << 40), dict(token_stride=1 << 40)])
def test_distillation_shapes_that_are_too_large(changes):
    assert distill_codes(distill(**changes)) == {TOO_LARGE}


def test_distillation_pointers():
    s, good = distill(), [16] * 6
    for at, bad in ((0, None), (0, 18), (1, None), (1, 18), (2, None), (2, 20), (3, 18), (4, 18)):
        assert solo.solo_distill(*good[:at], bad, *good[at + 1:5], s, stream=0, check=False) == BAD, (at, bad)
    for at, bad in ((0, None), (1, None), (2, 20), (3, None), (3, 18), (4, None), (4, 18), (5, None), (5, 18)):
        assert solo.solo_distill_grad(*good[:at], bad, *good[at + 1:], s, stream=0, check=False) == BAD, (at, bad)
    for at, bad in ((0, None), (1, None), (2, 20), (3, None), (3, 18), (4, 18), (5, None), (5, 18)):
        assert solo.solo_distill_with_grad(*good[:at], bad, *good[at + 1:], s, stream=0, check=False) == BAD, (at, bad)
    assert solo.solo_distill_grad(*good, distill(grad_stride=7), stream=0, check=False) == BAD
    assert solo.solo_distill_with_grad(*good, distill(grad_stride=7), stream=0, check=False) == BAD
    nothing = [None] * 6
    assert solo.solo_distill(*nothing[:5], distill(rows=0), stream=0) == solo.SOLO_OK
    assert solo.solo_distill_grad(*nothing, distill(rows=0), stream=0) == solo.SOLO_OK
    assert solo.solo_distill_with_grad(*nothing, distill(rows=0), stream=0) == solo.SOLO_OK
    for wrong in (None, 16, solo.solo_logits()):
        with pytest.raises((C.ArgumentError, TypeError)):
            solo.solo_distill(*good[:5], wrong, stream=0)


def test_distillation_handles_refuse_what_does_not_fit():
    plan = solo.SoloDistill(4, 8, 3, device="cpu")
    x, v, t, w = torch.zeros(4, 8), torch.zeros(4, 3), torch.zeros(4, 3, dtype=torch.int64), torch.zeros(4)
    for args in ((x[:, :7], v, t), (x, v[:3], t), (x, v, t[:, :2]), (x, v.t().contiguous().t(), t), (torch.zeros(5, 8), torch.zeros(5, 3), torch.zeros(5, 3).long())):
        with pytest.raises(ValueError):
            plan.forward(*args, stream=0)
    for args in ((x.half(), v, t), (x, v.double(), t), (x, v, t.short()), (x, v, t.float())):
        with pytest.raises(TypeError):
            plan.forward(*args, stream=0)
    for call in (plan.grad, plan.forward_grad):
        for args in ((x, v, t, w[:3], x), (x, v, t, w.double(), x), (x, v, t, w, x[:3]), (x, v, t, None, x)):
            with pytest.raises(ValueError):
                call(*args, stream=0)
        with pytest.raises(TypeError):
            call(x, v, t, w, x.bfloat16(), stream=0)
    with pytest.raises(ValueError, match="forward"):
        plan.grad(x, v, t, w, x, stream=0)
    for bad in (dict(top=0), dict(top=129), dict(top=3, rest=True, teacher_scale=2.0)):
        with pytest.raises(ValueError):
            solo.SoloDistill(4, 8, **bad, device="cpu")


# ---- sampling --------------------------------------------------------------------------------

def sample(**changes):
    return changed(solo.solo_sample_shape(4, 8, 8, 0, 64, 0, 0, 1.0, 1.0, 0.0, 0), changes)


@pytest.mark.parametrize("changes", [dict(dtype=2), dict(token_bits=8), dict(reserved=1), dict(reserved2=1), dict(temperature=-1.0), dict(temperature=math.nan),
                                     dict(top_p=math.nan), dict(min_p=math.nan), dict(stride=7)])
def test_sampling_shapes_that_are_refused(changes):
    assert solo.solo_sample(*[16] * 8, sample(**changes), stream=0, check=False) == BAD


@pytest.mark.parametrize("changes", [dict(cols=1 << 29, stride=1 << 29), dict(rows=1 << 35), dict(stride=1 << 40)])
def test_sampling_shapes_that_are_too_large(changes):
    assert solo.solo_sample(*[16] * 8, sample(**changes), stream=0, check=False) == TOO_LARGE


def test_sampling_pointers():
    s, good = sample(), [16] * 8
    for at, bad in ((0, None), (0, 18), (1, None), (1, 18), (2, 18), (3, 18), (4, 18), (5, 18), (6, None), (6, 20), (7, 18)):
        assert solo.solo_sample(*good[:at], bad, *good[at + 1:], s, stream=0, check=False) == BAD, (at, bad)
    assert solo.solo_sample(*[None] * 8, sample(rows=0), stream=0) == solo.SOLO_OK
    for wrong in (None, 16, solo.solo_logits()):
        with pytest.raises((C.ArgumentError, TypeError)):
            solo.solo_sample(*good, wrong, stream=0)


def test_sampling_handles_refuse_what_does_not_fit():
    plan = solo.SoloSampler(4, 8, device="cpu")
    x, u, k = torch.zeros(4, 8), torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    for args, more in (((x[:, :7], u), {}), ((x, u[:3]), {}), ((x, u.double()), {}), ((x, None), {}), ((torch.zeros(5, 8), torch.zeros(5)), {}), ((x, u), dict(top_k=u)),
                       ((x, u), dict(top_k=k.long())), ((x, u), dict(temperature=k)), ((x, u), dict(top_p=u[:2])), ((x, u), dict(min_p=torch.zeros(8)[::2]))):
        with pytest.raises(ValueError):
            plan.sample(*args, **more, stream=0)
    with pytest.raises(TypeError):
        plan.sample(x.half(), u, stream=0)
    for bad in (dict(temperature=-1.0), dict(temperature=math.nan), dict(top_p=math.nan), dict(min_p=math.nan)):
        with pytest.raises(ValueError):
            solo.SoloSampler(4, 8, **bad, device="cpu")


# ---- all of them -----------------------------------------------------------------------------

@pytest.mark.parametrize("native", (True, False))
def test_both_ways_into_the_library_take_the_same_arguments(tmp_path, native):
    b = fresh_binding(tmp_path, native)

    class Tensor:
        def data_ptr(self):
            return 16

    s = b.solo_layernorm_shape(0, 8, 8, 8, 8, 0, 1, 0, 0, 1e-5, 0)
    assert b.solo_layernorm(Tensor(), None, 16, Tensor(), None, s, stream=0) == b.SOLO_OK
    s.rows = 4
    assert b.solo_layernorm_grad(*[Tensor()] * 8, C.c_size_t(3), s, stream=0, check=False) == BAD
    with pytest.raises((C.ArgumentError, TypeError)):
        b.solo_layernorm_grad(*[Tensor()] * 8, 1.5, s, stream=0)
    s = b.solo_distill_shape(0, 8, 8, 8, 3, 3, 3, 0, 0, 64, 0, 0, 1.0, 1.0)
    assert b.solo_distill(Tensor(), 16, Tensor(), Tensor(), None, s, stream=0) == b.SOLO_OK
    assert b.solo_distill_grad(*[Tensor()] * 6, s, stream=0) == b.solo_distill_with_grad(*[Tensor()] * 6, s, stream=0) == b.SOLO_OK
    assert b.solo_sample(Tensor(), 16, None, Tensor(), None, None, 16, None, b.solo_sample_shape(0, 8, 8, 0, 32, 0, 0, 1.0, 1.0, 0.0, 0), stream=0) == b.SOLO_OK
    s.top = 0
    assert b.solo_distill_with_grad(*[Tensor()] * 6, s, stream=0, check=False) == BAD
