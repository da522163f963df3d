"""Ropes with more axes than turn pairs: positions [tokens][axes] go as they lie, whether the last axis turns a pair or not."""
import numpy as np
import pytest

import paper_2508_15601_amd as tm
from paper_2508_15601_amd import binding


class Library:
    """Stands for the native library: takes what it is given."""

    def tm_rope_create_axes(self, params, axes, axis):
        self.axes, self.axis = axes, None if axis is None else list(axis)
        return 1


@pytest.mark.parametrize("kw, axes, of_pair", [
    (dict(), 1, None), (dict(axes=1), 1, None), (dict(axis=[0, 1, 1, 0] * 2), 2, [0, 1, 1, 0] * 2), (dict(axis=[0, 1, 1, 0] * 2, axes=3), 3, [0, 1, 1, 0] * 2),
    (dict(axis=[0] * 8, axes=8), 8, [0] * 8), (dict(axis=[0] * 8), 1, [0] * 8)])
def test_axes_are_passed_on(monkeypatch, kw, axes, of_pair):
    lib = Library()
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    rope = tm.tm_rope_create(16, **kw)
    assert (lib.axes, lib.axis, rope.axes) == (axes, of_pair, axes)
    rope._h = 0                                                            # there is nothing to free


@pytest.mark.parametrize("kw, error", [(dict(axis=[0, 1] * 4, axes=1), tm.TmError), (dict(axes=2), tm.TmError), (dict(axis=[0] * 8, axes=9), tm.TmError), (dict(axis=[0] * 8, axes=0), tm.TmError),
                                       (dict(axis=[0] * 8, axes=-1), ValueError), (dict(axis=[0] * 8, axes=(1 << 32) + 1), ValueError), (dict(axis=[1 << 32] * 8), ValueError),
                                       (dict(axis=[0] * 7 + [-(1 << 32)]), ValueError)])
def test_axes_are_refused(kw, error):
    with pytest.raises(error, match="axes|axis"):
        tm.tm_rope_create(16, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("axes, other", [(3, 2), (8, 1)])
def test_an_axis_that_turns_no_pair(axes, other):
    """As with positions that leave it out, bit for bit, in all three calls that turn."""
    import torch
    axis = [i % other for i in range(64)]
    wide, narrow = tm.tm_rope_create(128, axis=axis, axes=axes), tm.tm_rope_create(128, axis=axis)
    assert tm.load_library().tm_rope_axes(wide.handle) == axes
    pos = torch.randint(-5, 1 << 30, (70, axes), device="cuda", dtype=torch.int32)
    few = pos[:, :other].contiguous() if other > 1 else pos[:, 0].contiguous()
    x = torch.randn(70, 10, 128, device="cuda").half()
    norm = tm.HeadNorm(torch.randn(128, device="cuda").half())
    out = []
    for rope, p in ((wide, pos), (narrow, few)):
        k, v, pairs = tm.tm_paged_pool(4, 2, 32, 8)
        cache = tm.tm_paged_create(k, v, pairs)
        y, z, q = torch.empty_like(x), torch.empty_like(x), torch.empty(70, 8, 128, dtype=torch.float16, device="cuda")
        tm.tm_rope_apply(x, p, rope, y)
        tm.tm_heads_apply(rope=rope, positions=p, Q=x, Q_out=z, q_norm=norm)
        batch = tm.PagedBatch(*(torch.tensor(a, dtype=torch.int32, device="cuda") for a in ([[2, 0, 3]], [0, 70], [0])))
        tm.tm_paged_append(cache, batch, x[:, :2], x[:, :2], rope=rope, Q=x[:, 2:], Q_out=q, q_norm=norm, k_norm=norm, positions=p)
        out.append((y, z, q, k, v, pairs))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    with pytest.raises(ValueError, match="axes"):
        tm.tm_rope_apply(x, few, wide, out[0][0])
    assert np.isfinite(out[0][0].float().cpu().numpy()).all()
