"""GPU parity of the append with norms and positions over tables most of whose rows have no new tokens: the same pages and queries, bit for bit, as over a table of the call's own rows."""
import sys

import numpy as np
import pytest

from test_gpu_heads import Heads, Pool, _dev, tm  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows, counts, past, max_count, q_heads, heads, rot, layout, axes, norm", [
    (300, [1, 1, 1, 1], [0, 31, 64, 90], 1, 8, 2, 128, "half", 1, "own"),                # by tokens
    (65, [5, 3, 8], [30, 0, 100], 8, 7, 1, 64, "interleaved", 3, "shared"),
    (300, [70, 1, 33], [5, 90, 31], 0, 28, 4, 128, "half", 3, "own"),                    # by runs
    (1000, [1, 40], [77, 0], 40, 6, 3, 96, "half", 1, "shared"),
    (200, [1, 2], [9, 60], 0, 5, 5, 0, "half", 1, "own"),                                # not turned
])
def test_rows_of_the_table_that_are_not_in_the_call(tm, bits, rows, counts, past, max_count, q_heads, heads, rot, layout, axes, norm):  # noqa: F811
    import torch
    print(f"append bits={bits} rows={rows} counts={counts} {q_heads}/{heads} rot={rot} {layout} axes={axes} {norm}", file=sys.stderr, flush=True)
    a, b = (Pool(tm, bits, 32, heads, counts, past, seed=rows, max_count=max_count) for _ in range(2))
    few = a.batch.table.cpu().numpy()
    rng = np.random.default_rng(rows)
    at = np.sort(rng.choice(rows, len(counts), replace=False))
    n, p, table = np.zeros(rows, np.int64), rng.integers(-5, 2000, rows), rng.integers(-1, a.k.shape[0] + 3, (rows, few.shape[1])).astype(np.int32)
    n[at], p[at], table[at] = counts, past, few                           # the other rows name pages of these, at any position
    b.batch = tm.PagedBatch(_dev(table), _dev((1 + np.concatenate([[0], np.cumsum(n)])).astype(np.int32)), _dev(p.astype(np.int32)), max_count=max_count)
    s = Heads(tm, a.tokens, q_heads, heads, 128, rot, layout, axes, norm, 1.0, norm == "own")
    V = torch.randn(a.tokens, heads, 128, device="cuda").half()
    out = []
    for pool in (a, b):
        q = torch.full((a.tokens, q_heads, 128), 7.0, dtype=torch.float16, device="cuda")
        tm.tm_paged_append(pool.cache, pool.batch, s.X["K"], V, rope=s.rope, Q=s.X["Q"], Q_out=q, q_norm=s.norm["Q"], k_norm=s.norm["K"], positions=None if axes == 1 else s.positions)
        out.append((q, *pool.contents()))
    assert all(torch.equal(x, y) for x, y in zip(*out))
    assert (out[1][0][[0, -2, -1]] == 7).all()                             # rows of no sequence, as they were
