"""GPU parity of attention in a sliding window where row tiles have 256 rows, whole and in pieces, alone and beside decoding sequences in one launch, and of tables with rows that are not in the
call; what the query hooks say of such calls.  Set-up and tolerance are those of test_gpu_paged_window.py."""
import numpy as np
import pytest

from test_gpu_paged_attn import _dev, _host
from test_gpu_paged_window import Window, tm  # noqa: F401

pytestmark = pytest.mark.gpu


def _plan(s):
    return s.tm.tm_get_paged_plan(s.cache, s.batch, s.tokens, s.q_heads, window=s.window, sinks=s.sinks)


def _form(s):
    return s.tm.tm_get_paged_form(s.cache, s.batch, s.tokens, s.q_heads, window=s.window, sinks=s.sinks)


def _window(tm, bits, window, sinks, page, heads, counts, positions, q_heads, **kw):  # noqa: F811
    return Window(tm, window, sinks, bits, page, heads, counts, positions, q_heads=q_heads, max_count=max(counts), max_len=max(c + p for c, p in zip(counts, positions)), seed=window, **kw)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("window, sinks, page, heads, q_heads, counts, positions, columns, pieces", [
    # alone: whole, then in pieces; tokens of one row tile, tokens over more than one (64 and 24 query heads)
    (150, 4, 64, 1, 64, [800], [300], 0, False),
    (97, 0, 32, 1, 64, [790, 30], [3, 1500], 16, False),
    (700, 4, 64, 1, 32, [1200], [7800], 0, True),
    (8000, 65, 32, 1, 24, [300], [9000], 0, True),
    (5000, 0, 1024, 1, 10, [500], [12000], 0, True),
    # decoding sequences in the same launch, by 8 and by 16 columns; a part of a 4-bit block to a page of 32
    (150, 40, 32, 1, 16, [1, 3300, 1, 0, 1], [500, 3, 90, 700, 2200], 16, False),
    (150, 0, 64, 1, 8, [1] * 3 + [6600] + [2], [500, 90, 0, 0, 1000], 8, False),
    (5000, 40, 32, 1, 8, [1] * 5 + [600], [3000, 90, 0, 1000, 31, 6000], 8, True),
    (4200, 3, 64, 1, 16, [1, 600, 1, 1], [9000, 6000, 5, 300], 16, True),
])
def test_tiles_of_256_rows(tm, bits, window, sinks, page, heads, q_heads, counts, positions, columns, pieces):  # noqa: F811
    s = _window(tm, bits, window, sinks, page, heads, counts, positions, q_heads)
    by, _, rows, most = _plan(s)
    launches, ctas, alone = _form(s)
    assert rows == 256 and by == columns and (most > 1) == pieces and launches == (2 if pieces else 1) and alone == bool(columns) and (ctas > 0) == bool(columns), (_plan(s), _form(s))
    s.check()


def test_tiles_of_128_rows_in_pieces(tm):  # noqa: F811
    """The windowed calls of test_a_chunk_in_pieces are cut, as the full ones that it asks about are."""
    for counts, q_heads, window in ([70], 4, 9000), ([17], 64, 5000), ([300], 4, 7000):
        for bits in (8, 4):
            s = Window(tm, window, 100, bits, 64, 1, counts, [12000], q_heads=q_heads, max_count=counts[0], max_len=12000 + counts[0], seed=counts[0])
            assert _plan(s)[2] == 128 and _plan(s)[3] > 1 and _form(s)[0] == 2, (_plan(s), _form(s))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("heads, q_heads, window, counts, positions", [(2, 16, 2048, [1] * 8 + [300], [5000, 3, 900, 4000, 70, 2500, 31, 0, 5000]), (4, 16, 300, [1, 90, 1], [700, 1000, 60]),
                                                                       (2, 8, 200, [1] * 20, list(range(0, 4000, 200)))])
@pytest.mark.parametrize("behind", [0, 3])
def test_rows_of_the_table_that_are_not_in_the_call(tm, bits, heads, q_heads, window, counts, positions, behind):  # noqa: F811
    """The same sequences among rows without new tokens: launched alike, the same bits, and rows behind the last token left as they were.  (Those may be tokens for all that the host knows, so
    with them a table of other sequences is one that may have three more that decode.)"""
    import torch
    s = _window(tm, bits, window, 4, 64, heads, counts, positions, q_heads, behind=behind)
    form, O = (_plan(s), _form(s)), s.run()
    rng = np.random.default_rng(7)
    for rows in (40, 64):
        at = np.sort(rng.choice(rows, len(counts), replace=False))
        n, p, table = np.zeros(rows, np.int64), rng.integers(0, 6000, rows), rng.integers(-1, s.k.shape[0], (rows, s.table.shape[1])).astype(np.int32)
        n[at], p[at], table[at] = counts, positions, s.table
        s.batch = tm.PagedBatch(_dev(table), _dev(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)), _dev(p.astype(np.int32)), max_count=s.batch.max_count, max_len=s.batch.max_len)
        if behind and rows == 40:
            form, O = (_plan(s), _form(s)), s.run()
        assert (_plan(s), _form(s)) == form
        assert torch.equal(s.run(), O)
    s.table, s.offsets, s.positions = table, np.concatenate([[0], np.cumsum(n)]), p.tolist()
    got, (want, A, S) = _host(O).astype(np.float64), s.want()
    there = ~np.isnan(want)
    assert (got[~there] == 7).all() and (~there).any() == bool(behind)
    sums = 2.0 ** -24 * (10 * 1039 if bits == 4 else 25 * 1151) * S
    assert (np.abs(got - want) <= 1.125 * 2.0 ** -11 * (np.abs(want) + A) + 2.0 ** -25 + sums)[there].all()


@pytest.mark.parametrize("rows", [65, 300])
def test_more_rows_of_the_table_than_a_wave_has_lanes(tm, rows):  # noqa: F811
    counts, positions = [1, 90, 1, 5], [700, 1000, 60, 300]
    rng = np.random.default_rng(rows)
    at = np.sort(rng.choice(rows, 4, replace=False))
    n, p = np.zeros(rows, np.int64), np.zeros(rows, np.int64)
    n[at], p[at] = counts, positions
    Window(tm, 300, 4, 8, 64, 1, n.tolist(), p.tolist(), q_heads=4, behind=1, max_count=90, max_len=1090, seed=rows).check()


def test_hooks_of_windows(tm):  # noqa: F811
    """A window that reaches as far as the table is no window; the hooks refuse what the call refuses."""
    s = Window(tm, 100, 4, 8, 64, 2, [100, 1], [700, 900], q_heads=8, max_count=100, cols=20, seed=4, taken=False)
    for hook in (tm.tm_get_paged_plan, tm.tm_get_paged_form):
        ask = lambda **kw: hook(s.cache, s.batch, s.tokens, s.q_heads, **kw)   # noqa: E731
        for window, sinks in ((s.cap, 0), ((1 << 31) - 1, 0), ((1 << 31) - 1, (1 << 31) - 1), (s.cap - 8, 8)):
            assert ask(window=window, sinks=sinks) == ask()
        for window, sinks, error in ((0, 0, tm.TmError), (-1, 0, tm.TmError), (5, -1, tm.TmError), (None, 4, ValueError), (1 << 31, 0, ValueError), (1, 1 << 40, ValueError)):
            with pytest.raises(error):
                ask(window=window, sinks=sinks)
