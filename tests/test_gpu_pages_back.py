"""Pages given back by thousands of rows (tm_paged_release) against plain Python: whole numbers, equal to the last."""
import time

import numpy as np
import pytest

from oracle import oracle_step as st
from test_gpu_pages import _dev, _host, tm  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch, wide, page, share, capacity", [
    (4096, 3, 32, 1.0, 20000),                                             # a CTA a row
    (4097, 3, 32, 1.0, 20000),                                             # rows by groups: the last one has one row
    (5000, 70, 64, 0.02, 9000),                                            # few rows give
    (6007, 130, 32, 0.5, 100000),                                          # more entries of a row than lanes; what the list has no room for is lost
    (65535, 2, 128, 0.7, 200000),
    (9000, 5, 1024, 0.0, 10),                                              # none does
])
def test_many_rows_give_back(tm, batch, wide, page, share, capacity):  # noqa: F811
    import torch
    rng = np.random.default_rng(batch)
    pool = batch * wide // (8 if page == 1024 else 1) + 5
    cache = tm.tm_paged_create(*tm.tm_paged_pool(pool, 1, page, 4))
    table = rng.integers(-2, pool + pool // 10, (batch, wide)).astype(np.int32)        # some name no page of the pool
    first = np.where(rng.random(batch) < share, rng.integers(-page, wide * page, batch), 1 << 30).astype(np.int32)
    last = (first.astype(np.int64) + rng.integers(-page, wide * page, batch)).clip(-(1 << 31), (1 << 31) - 1).astype(np.int32)
    pages = rng.integers(0, pool, capacity).astype(np.int32)
    for lo, hi, count in ((first, last, 7), (first, None, 0), (None, last, capacity - 1)):
        T, P, n = _dev(table), _dev(pages), torch.tensor([count], dtype=torch.int32, device="cuda")
        want = st.release(pages.tolist(), count, table, page, pool, lo, hi)
        free = tm.PageList(P, n)
        tm.tm_paged_release(cache, free, T, first=None if lo is None else _dev(lo), last=None if hi is None else _dev(hi))
        assert int(n) == want[1] and np.array_equal(_host(T), want[2])
        assert np.array_equal(_host(P), np.array(want[0], np.int32))


def test_rows_that_all_give_take_time_in_proportion(tm):  # noqa: F811
    """Eight times the rows, each of which gives a page back: not sixty-four times the work (a row that sums up all the others' counts makes it that)."""
    import torch
    took = []
    for batch in (8191, 65528):
        cache = tm.tm_paged_create(*tm.tm_paged_pool(batch, 1, 32, 4))
        ids = torch.arange(batch, dtype=torch.int32, device="cuda")
        T, P, n = torch.empty(batch, 2, dtype=torch.int32, device="cuda"), torch.empty(batch, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        best = 1e9
        for _ in range(20):
            T.copy_(ids[:, None].expand(batch, 2))
            T[:, 1] = -1
            n.zero_()
            torch.cuda.synchronize()
            t = time.perf_counter()
            tm.tm_paged_release(cache, tm.PageList(P, n), T)
            torch.cuda.synchronize()
            best = min(best, time.perf_counter() - t)
        assert int(n) == batch and torch.equal(P, ids.flip(0)) and (T == -1).all()
        took.append(best)
    assert took[1] < 16 * took[0] and took[1] < 400e-6, took
