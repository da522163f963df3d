"""Refusals of the entry points for norms of heads, positions of several axes and pages from lengths that end before a launch: arguments of the native binding
(TypeError, ValueError) and of the C ABI (negative status).  Runs without a GPU."""
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
LIST = tm.PageList(ints(4), ints(1))


@pytest.mark.parametrize("call, error", [
    (lambda: tm.tm_heads_apply(), ValueError),
    (lambda: tm.tm_heads_apply(Q=half(4, 2, 128)), ValueError),                                           # no Q_out
    (lambda: tm.tm_heads_apply(K_out=half(4, 2, 128)), ValueError),
    (lambda: tm.tm_heads_apply(Q=half(4, 2, 128), Q_out=half(4, 2, 128), k_norm=tm.HeadNorm()), ValueError),
    (lambda: tm.tm_heads_apply(rope=ROPE, Q=half(4, 2, 128), Q_out=half(4, 2, 128)), ValueError),         # no positions
    (lambda: tm.tm_heads_apply(positions=ints(4), Q=half(4, 2, 128), Q_out=half(4, 2, 128)), ValueError),
    (lambda: tm.tm_heads_apply(Q=half(4, 256), Q_out=half(4, 256)), ValueError),
    (lambda: tm.tm_heads_apply(Q=half(4, 2, 128), Q_out=half(4, 3, 128)), ValueError),
    (lambda: tm.tm_heads_apply(Q=half(4, 2, 128), Q_out=half(4, 2, 128), K=half(4, 2, 64), K_out=half(4, 2, 64)), ValueError),
    (lambda: tm.tm_heads_apply(Q=half(4, 2, 128), Q_out=half(4, 2, 128), K=half(5, 2, 128), K_out=half(5, 2, 128)), ValueError),
    (lambda: tm.tm_heads_apply(Q=half(4, 2, 128), Q_out=half(4, 2, 128)), TypeError),                     # host tensors
    (lambda: tm.tm_heads_apply(Q=[1.0], Q_out=half(4, 2, 128)), TypeError),
    (lambda: tm.tm_heads_apply(rope=ROPE, positions=ints(3), Q=half(4, 2, 128), Q_out=half(4, 2, 128)), ValueError),
    (lambda: tm.tm_heads_apply(rope=ROPE, positions=ints(4, 1), Q=half(4, 2, 128), Q_out=half(4, 2, 128)), ValueError),
    (lambda: tm.tm_rope_create(128, axis=[0] * 63), ValueError),
    (lambda: tm.tm_paged_assign(CACHE, LIST, BATCH, ints(2), ints(2)), ValueError),                       # neither slots nor tokens
    (lambda: tm.tm_paged_assign(CACHE, LIST, BATCH, ints(2), ints(2), slots=ints(4)), TypeError),
    (lambda: tm.tm_paged_assign(CACHE, LIST, BATCH, ints(2), ints(2), tokens=4), TypeError),              # host tensors
    (lambda: tm.tm_paged_assign(CACHE, LIST, BATCH, ints(2), ints(2), tokens=-1), ValueError),
    (lambda: tm.tm_paged_assign(CACHE, LIST, tm.PagedBatch(ints(6), ints(3), ints(2)), ints(2), ints(2), tokens=4), ValueError),
    (lambda: tm.tm_paged_release(CACHE, LIST, ints(6)), ValueError),
    (lambda: tm.tm_paged_release(CACHE, LIST, ints(2, 3)), TypeError),
    (lambda: tm.tm_paged_release(CACHE, LIST, None), TypeError),
])
def test_arguments_are_refused(call, error):
    with pytest.raises(error):
        call()


@pytest.mark.parametrize("axis", [[0] * 63 + [8], [-1] * 64, [0, -1] * 32])
def test_axes_are_refused(axis):
    with pytest.raises(tm.TmError, match="axes|axis"):
        tm.tm_rope_create(128, axis=axis)


class Norm(ctypes.Structure):
    _fields_ = [("weight", ctypes.c_void_p), ("weight_stride", ctypes.c_int64), ("eps", ctypes.c_double), ("offset", ctypes.c_double), ("centred", ctypes.c_int)]


class Rows(ctypes.Structure):
    _fields_ = [("X", ctypes.c_void_p), ("x_stride", ctypes.c_int64), ("Y", ctypes.c_void_p), ("y_stride", ctypes.c_int64), ("heads", ctypes.c_int), ("norm", ctypes.c_void_p)]


def test_c_entry_points_refuse_before_they_look_at_a_device():
    lib = tm.load_library()
    vp, i, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    fake = vp(4096)
    assert lib.tm_rope_create_axes(None, 1, None) is None and "null" in tm.tm_last_error()
    p = tm.binding.TmRopeParams(128, 0, 0, 10000.0, 1.0, 0.0, 0.0, 0.0, 0.0, None)
    for axes in (0, 9, 2):                                                # two without the axis of every pair
        assert lib.tm_rope_create_axes(ctypes.byref(p), axes, None) is None and "axes" in tm.tm_last_error()
    assert lib.tm_rope_axes(None) == -1
    lib.tm_heads_apply.argtypes = [vp, vp, vp, vp, i, i, vp]

    def heads(norm=None, dim=128, tokens=4, X=4096, xs=256, Y=8192, ys=256, n=2):
        r = Rows(X, xs, Y, ys, n, ctypes.cast(ctypes.pointer(norm), vp).value if norm is not None else None)
        return lib.tm_heads_apply(ctypes.byref(r), None, None, None, tokens, dim, None)

    assert lib.tm_heads_apply(None, None, None, None, 1, 128, None) == -1 and "neither" in tm.tm_last_error()
    assert heads() in (-2, -3)                                            # nothing to refuse but the device
    for kw, text in [(dict(dim=12), "head_dim"), (dict(dim=0), "head_dim"), (dict(dim=264), "head_dim"), (dict(tokens=-1), "tokens"), (dict(X=None), "null"), (dict(Y=None), "null"),
                     (dict(X=4104), "aligned"), (dict(xs=248), "stride"), (dict(ys=260), "stride"), (dict(n=0), "heads"), (dict(n=65536), "heads"),
                     (dict(X=4096, Y=4096, ys=512), "equal strides"), (dict(norm=Norm(None, 0, 0.0, 0.0, 0)), "eps"), (dict(norm=Norm(None, 0, float("inf"), 0.0, 0)), "eps"),
                     (dict(norm=Norm(None, 0, 1e-6, float("nan"), 0)), "offset"), (dict(norm=Norm(None, 0, 1e-6, 0.0, 2)), "centred"),
                     (dict(norm=Norm(4104, 0, 1e-6, 0.0, 0)), "aligned"), (dict(norm=Norm(4096, 120, 1e-6, 0.0, 0)), "weight_stride"),
                     (dict(norm=Norm(4096, -128, 1e-6, 0.0, 0)), "weight_stride"), (dict(norm=Norm(4096, 132, 1e-6, 0.0, 0)), "weight_stride")]:
        assert heads(**kw) == -1 and text in tm.tm_last_error(), (kw, tm.tm_last_error())
    assert heads(tokens=0, X=None, Y=None) == 0
    lib.tm_paged_append_heads.argtypes = [vp, vp, vp, i64, vp, i64, vp, vp, i64, vp, i64, i, vp]
    assert lib.tm_paged_append_heads(None, fake, fake, 256, fake, 256, fake, None, 0, None, 0, 0, None) == -1 and "cache" in tm.tm_last_error()
    lib.tm_paged_assign.argtypes = [vp] * 4
    assert lib.tm_paged_assign(None, None, None, None) == -1 and "step" in tm.tm_last_error()
    lib.tm_paged_release.argtypes = [vp, vp, vp, i, i, vp, vp, vp]
    assert lib.tm_paged_release(None, fake, fake, 1, 1, None, None, None) == -1 and "cache" in tm.tm_last_error()
