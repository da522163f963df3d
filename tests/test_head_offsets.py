"""Norms of heads with offsets of any size: a head of zeros is 0 whatever its weights are, and offsets whose product with 1 / sqrt(eps) would leave the range of 64 bits are refused."""
import ctypes

import pytest

import paper_2508_15601_amd as tm
from test_step_calls import Norm, Rows


@pytest.mark.parametrize("offset, fine", [(0.0, True), (-1e150, True), (1e150, True), (1.001e150, False), (-1e158, False), (1e308, False), (float("inf"), False), (float("nan"), False)])
def test_offsets_out_of_range_are_refused(offset, fine):
    lib = tm.load_library()
    vp, i = ctypes.c_void_p, ctypes.c_int
    lib.tm_heads_apply.argtypes = [vp, vp, vp, vp, i, i, vp]
    norm = Norm(None, 0, 1e-300, offset, 0)
    rows = Rows(None, 256, None, 256, 2, ctypes.cast(ctypes.pointer(norm), vp).value)
    rc = lib.tm_heads_apply(ctypes.byref(rows), None, None, None, 0, 128, None)       # no tokens: arguments are all that is looked at
    assert rc == (0 if fine else -1), tm.tm_last_error()
    if not fine:
        assert "offset" in tm.tm_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("centred", [False, True])
@pytest.mark.parametrize("offset", [1e150, -1e150, 65504.0])
def test_a_head_of_zeros_is_zero(offset, centred):
    """With the smallest eps and the largest offsets, turned or not, alone and in the append; a head of anything else is its sign times infinity where that is beyond fp16."""
    import torch
    x = torch.zeros(3, 6, 128, dtype=torch.float16, device="cuda")
    x[:, 5] = torch.randn(3, 128, device="cuda").half()
    y, pos = torch.full_like(x, 7.0), torch.tensor([0, 5, 90], dtype=torch.int32, device="cuda")
    norm = tm.HeadNorm(None, eps=1e-300, offset=offset, centred=centred)
    for rope in (None, tm.tm_rope_create(128, amplitude=1e4), tm.tm_rope_create(64, layout=tm.TM_ROPE_INTERLEAVED)):
        tm.tm_heads_apply(rope=rope, positions=None if rope is None else pos, Q=x, Q_out=y, q_norm=norm)
        assert (y[:, :5] == 0).all() and not y[:, 5].isnan().any()
        if offset != 65504.0 and rope is None and not centred:
            assert torch.equal(y[:, 5], torch.where(x[:, 5] == 0, x[:, 5], torch.sign(x[:, 5]) * (torch.inf if offset > 0 else -torch.inf)))
        for count in (1, 3):                                               # by tokens and by runs
            pool = tm.tm_paged_pool(3, 6, 32, 8)
            batch = tm.PagedBatch(*(torch.tensor(a, dtype=torch.int32, device="cuda") for a in (([[0], [1], [2]], [0, 1, 2, 3], [0, 5, 9]) if count == 1 else ([[1]], [0, 3], [0]))), max_count=count % 3)
            out = torch.full_like(x, 7.0)
            cache = tm.tm_paged_create(*pool)
            tm.tm_paged_append(cache, batch, x, x, rope=rope, Q=x, Q_out=out, q_norm=norm, k_norm=norm)
            K, V = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
            tm.tm_paged_read(cache, batch, K, V)
            assert (out[:, :5] == 0).all() and (K[:, :5] == 0).all() and not out[:, 5].isnan().any()
