"""How a tm_paged_attn call is launched (tm_get_paged_form) at the shapes whose kernels the parity tests mean to run, further parity in forms that differ by that alone, and a prompt
followed by decoding steps beside the contiguous cache, what is stored included."""
import numpy as np
import pytest

from oracle import oracle_attn as oa
from oracle import oracle_paged as op
from test_gpu_paged_attn import SCALE, Setup, _dev, _host, _lengths, tm  # noqa: F401

pytestmark = pytest.mark.gpu


def _form(s):
    return s.tm.tm_get_paged_form(s.cache, s.batch, s.tokens, s.q_heads)


@pytest.mark.parametrize("bits, page, heads, q_heads, batch, longest, count, max_len, launches, ctas, alone", [
    # more segments (sequence, KV head, column tile) than compute units: every wave by itself; 8-bit codes from four of them on
    (4, 32, 8, 32, 40, 700, 1, 0, 1, 256, True),
    (4, 64, 8, 8, 40, 3600, 1, 0, 1, 256, True),
    (4, 64, 4, 48, 70, 300, 1, 0, 1, 256, True),
    (4, 128, 8, 40, 34, 500, 5, 0, 1, 256, True),
    (4, 32, 2, 6, 131, 400, 2, 0, 1, 256, True),
    (8, 64, 16, 32, 64, 1500, 1, 1501, 1, 256, True),
    (8, 32, 16, 160, 66, 300, 1, 0, 1, 256, True),
    (8, 64, 16, 32, 64, 200, 3, 0, 1, 256, True),
    (8, 64, 8, 32, 33, 500, 1, 501, 1, 512, False),                        # short contexts: two CTAs a compute unit
    (8, 32, 4, 40, 90, 700, 1, 701, 1, 512, False),
    (8, 32, 4, 40, 90, 700, 1, 0, 1, 256, False),                          # the same without the hint
    (4, 32, 8, 16, 32, 333, 1, 0, 1, 256, False),                          # as many segments as compute units
    (8, 32, 8, 16, 130, 333, 1, 0, 1, 256, True),
])
def test_many_segments(tm, bits, page, heads, q_heads, batch, longest, count, max_len, launches, ctas, alone):  # noqa: F811
    counts = [count] * batch
    counts[1] = 0
    s = Setup(tm, bits, page, heads, counts, _lengths(batch, longest, page), q_heads=q_heads, before=1, behind=1, max_count=count, max_len=max_len, seed=batch)
    assert _form(s) == (launches, ctas, alone)
    s.check()


@pytest.mark.parametrize("bits", [8, 4])
def test_rows_and_columns(tm, bits):  # noqa: F811
    """Long new tokens alone; beside short ones in one launch; in two, where a table is wider than a wave's count of blocks allows.  One launch more where contexts are cut."""
    s = Setup(tm, bits, 64, 8, [400], [0], q_heads=8, seed=400)
    assert _form(s)[1:] == (0, False) and _form(s)[0] in (1, 2)
    s = Setup(tm, bits, 64, 8, [1, 100, 3], [200, 900, 70], q_heads=32, seed=5, max_count=100, max_len=1000)
    launches, ctas, alone = _form(s)
    assert launches == 2 and ctas in (128, 176) and alone
    O = s.check((True, True, True, True))
    s.table = np.pad(s.table, ((0, 0), (0, 2600000 - s.table.shape[1])), constant_values=-1)
    s.batch = tm.PagedBatch(_dev(s.table), s.batch.offsets, s.batch.positions, max_count=100, max_len=1000)
    assert _form(s) == (3, 256, False)
    wide = s.check((True, True, True, True))
    assert not np.isnan(_host(O)).any() and not np.isnan(_host(wide)).any()
    s.batch = tm.PagedBatch(s.batch.table, s.batch.offsets, s.batch.positions, max_count=100, max_len=300)
    assert _form(s) == (2, 256, False)                                     # short contexts are not cut
    s.check((True, True, True, 1))


def test_widest_tables(tm):  # noqa: F811
    """The bound on the work of a call that tm_paged.h states: tables of 2^28 tokens for 64 decoding sequences of 8 KV heads and 4 query heads each, and no wider ones."""
    import torch
    cache = tm.tm_paged_create(*tm.tm_paged_pool(2, 8, 1024, 8))
    offsets, positions = torch.arange(65, dtype=torch.int32, device="cuda"), torch.arange(64, dtype=torch.int32, device="cuda")
    Q = torch.randn(64, 32, 128, device="cuda").half()
    for columns in (1 << 18, 1 << 19):
        batch = tm.PagedBatch(torch.full((64, columns), -1, dtype=torch.int32, device="cuda"), offsets, positions)
        O = torch.full_like(Q, 7.0)
        if columns == 1 << 18:
            tm.tm_paged_attn(Q, cache, batch, O, SCALE)
            assert (O == 0).all()                                          # no page of theirs is there
        else:
            for call in (lambda: tm.tm_paged_attn(Q, cache, batch, O, SCALE), lambda: tm.tm_get_paged_plan(cache, batch, 64, 32), lambda: tm.tm_get_paged_form(cache, batch, 64, 32)):
                with pytest.raises(tm.TmError, match="too much work"):
                    call()
            assert (O == 7).all()


def test_refusals(tm):  # noqa: F811
    s = Setup(tm, 8, 32, 2, [4], [0], q_heads=4)
    with pytest.raises(tm.TmError, match="q_heads"):
        tm.tm_get_paged_form(s.cache, s.batch, 4, 3)
    with pytest.raises(ValueError, match="tokens"):
        tm.tm_get_paged_form(s.cache, s.batch, -1, 4)
    s.cache.close()
    with pytest.raises(ValueError, match="freed"):
        tm.tm_get_paged_form(s.cache, s.batch, 4, 4)


@pytest.mark.parametrize("bits", [8, 4])
def test_serving_steps_store_what_the_contiguous_cache_does(tm, bits):  # noqa: F811
    """A prompt in chunks and decoding steps after it, two sequences: after every step the pages hold what tm_kv_append stores, bit for bit, and both attentions are within their
    tolerance of the oracle over it (the header of test_gpu_paged_attn.py), value by value."""
    import torch
    heads, q_heads, page, cap = 2, 8, 64, 384
    k, v, pairs = tm.tm_paged_pool(12, heads, page, bits)
    cache, slab = tm.tm_paged_create(k, v, pairs), tm.tm_kv_create(2, heads, cap, bits)
    rows = np.random.default_rng(0).permutation(12).reshape(2, 6).astype(np.int32)
    table, at, past = _dev(rows), torch.zeros(2, dtype=torch.int32, device="cuda"), 0
    torch.manual_seed(bits)
    for n in (100, 37, 1, 1, 8, 1):
        Q, K, V = (torch.randn(2, n, h, 128, device="cuda").half() for h in (q_heads, heads, heads))
        batch = tm.PagedBatch(table, torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda"), at, max_count=n)
        tm.tm_paged_append(cache, batch, K.view(2 * n, heads, 128), V.view(2 * n, heads, 128))
        tm.tm_kv_append(slab, K, V, at)
        arrays = op.unpack_pool(_host(k), _host(v), _host(pairs))
        for got, want in zip(arrays, oa.kv_cache_unpack(*tm.tm_kv_download(slab), 2, heads, cap, bits)):
            for b in range(2):
                joined = np.concatenate([got[p] for p in rows[b]], axis=1)[:, :past + n]
                assert np.array_equal(joined, want[b, :, :past + n])
        want, A = op.attention(_host(Q).reshape(2 * n, q_heads, 128), arrays, rows, [0, n, 2 * n], [past, past], SCALE)
        O, P = torch.empty(2 * n, q_heads, 128, dtype=torch.float16, device="cuda"), torch.empty(2, n, q_heads, 128, dtype=torch.float16, device="cuda")
        tm.tm_paged_attn(Q.view(2 * n, q_heads, 128), cache, batch, O, SCALE)
        tm.tm_attn_prefill(Q, slab, at, P, SCALE)
        for out in (_host(O), _host(P).reshape(O.shape)):
            assert (np.abs(out.astype(np.float64) - want) <= 1.125 * 2.0 ** -11 * (np.abs(want) + A) + 2.0 ** -25).all()
        at += n
        past += n
    slab.close()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("counts, positions", [([1, 1], [600, 40]), ([100], [200])])
@pytest.mark.parametrize("size", [1e-2, 1e-4])
def test_values_next_to_fp16s_smallest(tm, bits, counts, positions, size):  # noqa: F811
    """Values so small that a probability times a value's scale is no normal fp16 number: its rounding is then off by 2^-25 and not by 2^-11 of it.  A value meets it (q - z) times, and the
    denominator is at least the sum of the probabilities relative to the largest.  Sums that carry the codes' bias add 24 steps of 2^-24 of up to 1279 scales, as where V^ is 0."""
    import torch
    s = Setup(tm, bits, 32, 1, counts, positions, q_heads=4, seed=11)
    total = int(s.positions[0]) + counts[0] + (s.positions[1] + counts[1] if len(counts) > 1 else 0)
    lens = [n + p for n, p in zip(counts, positions)]
    fill = tm.PagedBatch(s.batch.table, _dev(np.cumsum([0] + lens).astype(np.int32)), torch.zeros(len(counts), dtype=torch.int32, device="cuda"))
    g = torch.Generator(device="cuda")
    g.manual_seed(12)
    K, V = (torch.randn(total, 1, 128, generator=g, device="cuda") for _ in range(2))
    tm.tm_paged_append(s.cache, fill, K.half(), (V * size).half())
    O = _host(s.run()).astype(np.float64)
    want, A = s.want()
    arrays = op.unpack_pool(_host(s.k), _host(s.v), _host(s.pairs))
    Q = _host(s.Q).astype(np.float64)
    for b, (n, p) in enumerate(zip(counts, positions)):
        Kb, _, ok = op.gather(arrays, s.table[b], p + n)
        assert ok.all()
        t = np.arange(p + n)
        page, slot = s.table[b, t // s.page], t % s.page
        steps = np.abs(arrays[3][page, 0, slot].astype(np.float64) - arrays[5][page, 0, slot].astype(np.float64)[:, None])          # |q - z| [tokens][128]
        scale = arrays[4][page, 0, slot].astype(np.float64).max()
        for i in range(n):
            row = int(s.offsets[b]) + i
            x = Kb[:p + i + 1, 0] @ Q[row].T * SCALE                       # [tokens][heads]
            L = np.exp(x - x.max(0)).sum(0)
            bound = 1.125 * 2.0 ** -11 * (np.abs(want[row]) + A[row]) + 2.0 ** -25 * steps[:p + i + 1].sum(0)[None] / L[:, None] + 24 * 2.0 ** -24 * 1279 * scale + 2.0 ** -25
            assert (np.abs(O[row] - want[row]) <= bound).all(), (b, i)
