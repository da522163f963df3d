"""Refusals of the paged cache's and the rotary positions' entry points that end before a launch: arguments of the native binding (TypeError, ValueError)
and of the C ABI (negative status).  Runs without a GPU."""
import ctypes
import types

import pytest
import torch

import paper_2508_15601_amd as tm


def half(*shape):
    return torch.zeros(shape, dtype=torch.float16)


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


CACHE = types.SimpleNamespace(_h=0, kv_heads=2)
ROPE = types.SimpleNamespace(_h=0)
BATCH = tm.PagedBatch(ints(2, 3), ints(3), ints(2))


@pytest.mark.parametrize("call, error", [
    (lambda: tm.tm_rope_apply([0.0], ints(1), ROPE, half(1, 1, 128)), TypeError),
    (lambda: tm.tm_rope_apply(half(4, 2, 128), ints(4), ROPE, half(4, 2, 128)), TypeError),               # host tensors
    (lambda: tm.tm_rope_apply(half(4, 2, 128), ints(3), ROPE, half(4, 2, 128)), ValueError),
    (lambda: tm.tm_rope_apply(half(4, 2, 128), ints(4, 1), ROPE, half(4, 2, 128)), ValueError),
    (lambda: tm.tm_rope_apply(half(4, 256), ints(4), ROPE, half(4, 256)), ValueError),
    (lambda: tm.tm_rope_apply(half(4, 2, 128), ints(4), ROPE, half(4, 1, 128)), ValueError),
    (lambda: tm.tm_paged_append(CACHE, BATCH, half(4, 2, 64), half(4, 2, 64)), ValueError),
    (lambda: tm.tm_paged_append(CACHE, BATCH, half(4, 3, 128), half(4, 3, 128)), ValueError),             # another number of heads
    (lambda: tm.tm_paged_append(CACHE, BATCH, half(4, 2, 128), half(3, 2, 128)), ValueError),
    (lambda: tm.tm_paged_append(CACHE, BATCH, half(4, 2, 128), half(4, 2, 128)), TypeError),              # host tensors
    (lambda: tm.tm_paged_append(CACHE, tm.PagedBatch(ints(6), ints(3), ints(2)), half(4, 2, 128), half(4, 2, 128)), ValueError),
    (lambda: tm.tm_paged_append(CACHE, tm.PagedBatch(ints(2, 3), ints(2), ints(2)), half(4, 2, 128), half(4, 2, 128)), ValueError),
    (lambda: tm.tm_paged_append(CACHE, tm.PagedBatch(ints(2, 3), ints(3), ints(3)), half(4, 2, 128), half(4, 2, 128)), ValueError),
    (lambda: tm.tm_paged_append(CACHE, tm.PagedBatch(None, ints(3), ints(3)), half(4, 2, 128), half(4, 2, 128)), TypeError),
    (lambda: tm.tm_paged_read(CACHE, BATCH, half(4, 2, 128), half(4, 2, 64)), ValueError),
    (lambda: tm.tm_paged_read(CACHE, BATCH, half(4, 2, 128), half(4, 2, 128)), TypeError),
    (lambda: tm.tm_paged_create(ints(1), ints(1), half(1)), ValueError),
    (lambda: tm.tm_paged_create(*tm.tm_paged_pool(2, 1, 32, 8, device="cpu")), TypeError),                # host tensors
    (lambda: tm.tm_rope_create(128, frequencies=[1.0] * 63), ValueError),
])
def test_arguments_are_refused(call, error):
    with pytest.raises(error):
        call()


@pytest.mark.parametrize("params, text", [
    (dict(rot_dim=0), "rot_dim"), (dict(rot_dim=24), "rot_dim"), (dict(rot_dim=272), "rot_dim"), (dict(layout=2), "layout"), (dict(layout=-1), "layout"),
    (dict(scaling=5), "scaling"), (dict(base=1.0), "out of range"), (dict(base=float("nan")), "out of range"), (dict(base=float("inf")), "out of range"),
    (dict(scaling=tm.TM_ROPE_LINEAR, factor=0.5), "out of range"), (dict(scaling=tm.TM_ROPE_BASE, factor=float("inf")), "out of range"),
    (dict(scaling=tm.TM_ROPE_WAVELENGTH, factor=8.0, low=1.0, high=4.0), "out of range"),                 # no original length
    (dict(scaling=tm.TM_ROPE_WAVELENGTH, factor=8.0, original_len=4096, low=4.0, high=4.0), "out of range"),
    (dict(scaling=tm.TM_ROPE_RAMP, factor=8.0, original_len=4096, low=0.0, high=4.0), "out of range"),
    (dict(amplitude=float("nan")), "out of range"), (dict(frequencies=[float("nan")] * 64), "out of range"), (dict(frequencies=[1e9] * 64), "out of range"),
])
def test_rope_parameters_are_refused(params, text):
    with pytest.raises(tm.TmError, match=text):
        tm.tm_rope_create(**params)


def test_c_entry_points_refuse_before_they_look_at_a_device():
    lib = tm.load_library()
    fake, vp, i, i64 = ctypes.c_void_p(4096), ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    assert lib.tm_rope_create(None) is None and "null" in tm.tm_last_error()
    assert lib.tm_rope_frequencies(None, None, None) == -1
    lib.tm_rope_free(None)
    lib.tm_rope_apply.argtypes = [vp, i64, vp, vp, vp, i64, i, i, i, vp]
    assert lib.tm_rope_apply(fake, 128, fake, None, fake, 128, 1, 1, 128, None) == -1 and "rope" in tm.tm_last_error()
    need = lib.tm_paged_workspace_bytes()
    for args, text in [((None, fake, fake, 4, 2, 32, 8, fake, need), "null"), ((fake, fake, fake, 4, 2, 32, 8, None, need), "null"),
                       ((vp(4100), fake, fake, 4, 2, 32, 8, fake, need), "misaligned"), ((fake, fake, fake, 4, 2, 32, 8, vp(4112), need), "misaligned"),
                       ((fake, fake, fake, 0, 2, 32, 8, fake, need), "pages"), ((fake, fake, fake, 4, 0, 32, 8, fake, need), "heads"),
                       ((fake, fake, fake, 4, 2, 16, 8, fake, need), "power of two"), ((fake, fake, fake, 4, 2, 96, 8, fake, need), "power of two"),
                       ((fake, fake, fake, 4, 2, 2048, 8, fake, need), "power of two"), ((fake, fake, fake, 4, 2, 32, 16, fake, need), "bits"),
                       ((fake, fake, fake, 4, 2, 32, 8, fake, need - 1), "workspace")]:
        assert lib.tm_paged_create(*args) is None and text in tm.tm_last_error(), (args, tm.tm_last_error())
    lib.tm_paged_free(None)
    lib.tm_paged_append.argtypes = [vp, vp, vp, i64, vp, i64, vp, vp, i64, vp, i64, i, vp]
    assert lib.tm_paged_append(None, fake, fake, 256, fake, 256, None, None, 0, None, 0, 0, None) == -1 and "cache" in tm.tm_last_error()
    lib.tm_paged_read.argtypes = [vp] * 5
    assert lib.tm_paged_read(None, fake, fake, fake, None) == -1
