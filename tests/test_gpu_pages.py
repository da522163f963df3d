"""Pages from lengths on the GPU (tm_paged_assign, tm_paged_release) against plain Python: whole numbers, equal to the last."""
import sys

import numpy as np
import pytest

from oracle import oracle_step as st

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tm():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_2508_15601_amd as tm
    tm.load_library()
    return tm


def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _host(t):
    import torch
    torch.cuda.synchronize()
    return t.cpu().numpy()


class Rows:
    """Rows with lens tokens each, in pages of no order; `spare` pages on a list, of which the first `free` count."""

    def __init__(self, tm, lens, page, max_pages, spare, free=None, seed=0):
        rng = np.random.default_rng(seed)
        self.tm, self.page = tm, page
        have = [min(-(-max(n, 0) // page), max_pages) for n in lens]
        self.pool = sum(have) + spare + 1
        ids = rng.permutation(self.pool).astype(np.int32)
        self.table = np.full((len(lens), max_pages), -1, np.int32)
        done = 0
        for b, n in enumerate(have):
            self.table[b, :n] = ids[done:done + n]
            done += n
        self.pages, self.count = ids[done:done + spare].copy(), spare if free is None else free
        self.lens = np.array(lens, np.int32)
        self.cache = tm.tm_paged_create(*tm.tm_paged_pool(self.pool, 1, page, bits=4))
        self.T = _dev(self.table)
        self.list = tm.PageList(_dev(self.pages), _dev(np.array([self.count], np.int32)))

    def batch(self):
        import torch
        B = len(self.lens)
        return self.tm.PagedBatch(self.T, torch.full((B + 1,), -7, dtype=torch.int32, device="cuda"), torch.full((B,), -7, dtype=torch.int32, device="cuda"))

    def check(self, counts, tokens=None, room=3):
        """One call, not in place; returns what the oracle says."""
        import torch
        total = int(np.maximum(np.array(counts, np.int64), 0).sum())
        tokens = total + room if tokens is None else tokens
        want = st.assign(self.pages.tolist(), self.count, self.lens, counts, self.table, self.page, self.pool, tokens)
        slots = torch.full((tokens,), -9, dtype=torch.int64, device="cuda")
        lens_out, short, left = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for n in (len(self.lens), len(self.lens), 1))
        batch, lens, new = self.batch(), _dev(self.lens), _dev(np.array(counts, np.int32))
        self.tm.tm_paged_assign(self.cache, self.list, batch, lens, new, slots=slots, short=short, lens_out=lens_out, left=left)
        got = dict(table=_host(self.T), offsets=_host(batch.offsets), positions=_host(batch.positions), lens=_host(lens_out), lacking=_host(short), left=int(left))
        for k, v in got.items():
            assert np.array_equal(v, want[k]), (k, v, want[k])
        expected = np.full(tokens, -9, np.int64)
        for t, slot in want["slots"].items():
            expected[t] = slot
        assert np.array_equal(_host(slots), expected)
        assert np.array_equal(_host(self.list.pages), self.pages) and int(self.list.count) == self.count and np.array_equal(_host(lens), self.lens)
        # in place, without what may be left out
        again = Rows.__new__(Rows)
        again.__dict__.update(self.__dict__)
        T2, count = _dev(self.table), self.list.count.clone()
        b2 = self.tm.PagedBatch(T2, torch.empty_like(batch.offsets), torch.empty_like(batch.positions))
        self.tm.tm_paged_assign(self.cache, self.tm.PageList(self.list.pages, count), b2, lens, new, tokens=tokens)
        assert torch.equal(T2, self.T) and torch.equal(b2.offsets, batch.offsets) and torch.equal(lens, lens_out) and torch.equal(count, left)
        return want


CASES = [
    # lens, counts, page, max_pages, spare pages
    ([0], [1], 32, 1, 1),
    ([0], [0], 32, 1, 1),
    ([31, 32, 33, 0], [1, 1, 1, 1], 32, 3, 9),
    ([63, 64, 65], [0, 130, 2], 64, 5, 9),
    ([5, 5], [1000, 3], 32, 40, 100),
    ([0, 0, 0, 0], [64, 64, 64, 1], 64, 4, 2),                             # too few: rows from the third on
    ([10, 32, 20], [5, 1, 5], 32, 4, 0),                                   # none at all: rows that need none are served
    ([90, 96, 500], [20, 7, 1], 32, 3, 8),                                 # rows that reach the end of the table, and beyond it
    ([-5, 3], [4, -8], 32, 2, 4),                                          # lengths and counts below zero
    ([1000, 0], [2000000000, 2000000000], 1024, 8, 40),                    # more than the packed arrays hold
]


@pytest.mark.parametrize("lens, counts, page, max_pages, spare", CASES)
def test_assign(tm, lens, counts, page, max_pages, spare):
    total = sum(max(c, 0) for c in counts)
    Rows(tm, lens, page, max_pages, spare).check(counts, tokens=5000 if total > 100000 else None)


@pytest.mark.parametrize("batch", [1, 63, 64, 65, 256, 257, 1000, 1024, 1025, 2048, 4096, 4097, 9001])
@pytest.mark.parametrize("kind", ["decode", "mixed", "scarce"])
def test_assign_many_rows(tm, batch, kind):
    print(f"assign batch={batch} {kind}", file=sys.stderr, flush=True)
    rng = np.random.default_rng(batch)
    lens = rng.integers(0, 700, batch)
    counts = rng.choice([0, 1, 1, 1], batch) if kind == "decode" else np.where(rng.random(batch) < 0.1, rng.integers(0, 400, batch), rng.choice([0, 1], batch))
    need = int(sum(-(-(n + c) // 32) - -(-n // 32) for n, c in zip(lens.tolist(), counts.tolist())))
    Rows(tm, lens.tolist(), 32, 40, max(need, 1), free=need * 2 // 3 if kind == "scarce" else None, seed=batch).check(counts.tolist())


@pytest.mark.parametrize("tokens", [0, 1, 30, 64, 100])
@pytest.mark.parametrize("batch", [3, 1500, 5000])
def test_packed_arrays_that_are_too_small(tm, tokens, batch):
    Rows(tm, [20] * batch, 32, 4, 2 * batch).check([33] * batch, tokens=tokens)


@pytest.mark.parametrize("count", [-3, 0, 7, 1000])
def test_lists_count_is_limited(tm, count):
    Rows(tm, [0] * 9, 32, 2, 8, free=count).check([1] * 9)


def test_list_of_pages_that_the_pool_does_not_have(tm):
    """They become entries that name no page; their tokens have no slot."""
    r = Rows(tm, [0, 31], 32, 3, 4)
    r.pages[:] = [-1, 1 << 30, r.pool, 0]
    r.list.pages.copy_(_dev(r.pages))
    r.check([40, 2])


RELEASES = [
    # lens, first, last
    ([0, 100, 333], None, None),                                           # whole rows
    ([100, 333, 64], [33, 320, 64], None),                                 # behind a length
    ([300, 64, 1000], None, [299, 64, 10]),                                # before one
    ([300, 640, 1000], [4, 4, 64], [299, 63, 500]),                        # between first tokens and a window
    ([300, 640], [-5, 2000000000], [-1, 2000000000]),
]


@pytest.mark.parametrize("lens, first, last", RELEASES)
@pytest.mark.parametrize("page", [32, 64])
def test_release(tm, lens, first, last, page):
    import torch
    r = Rows(tm, lens, page, 40, 5, free=3)
    r.pages = np.concatenate([r.pages, np.full(12, -5, np.int32)])         # a list that holds some of them, not all
    r.list.pages = _dev(r.pages)
    r.table[0, 30], r.table[-1, 2] = r.pool, -2                            # no pages of the pool
    r.T = _dev(r.table)
    want = st.release(r.pages.tolist(), 3, r.table, page, r.pool, first, last)
    ints = lambda x: None if x is None else _dev(np.array(x, np.int32))  # noqa: E731
    left = torch.zeros(1, dtype=torch.int32, device="cuda")
    tm.tm_paged_release(r.cache, r.list, r.T, first=ints(first), last=ints(last), left=left)
    assert int(left) == want[1] and _host(r.list.pages).tolist() == want[0] and np.array_equal(_host(r.T), want[2]) and int(r.list.count) == 3
    tm.tm_paged_release(r.cache, r.list, r.T, first=ints(first), last=ints(last))          # there is nothing left: in place
    assert int(r.list.count) == 3


@pytest.mark.parametrize("batch, wide", [(1, 3000), (300, 70), (2000, 9)])
def test_what_goes_back_comes_again(tm, batch, wide):
    """Assigned and given back, the list is what it was; assigned again, so is the table."""
    import torch
    rng = np.random.default_rng(wide)
    lens = rng.integers(0, 32 * wide // 2, batch)
    counts = rng.integers(0, 32 * wide // 2, batch)
    r = Rows(tm, lens.tolist(), 32, wide, int(sum(-(-(n + c) // 32) - -(-n // 32) for n, c in zip(lens.tolist(), counts.tolist()))) + 4, seed=1)
    lens, counts, total = _dev(r.lens), _dev(counts.astype(np.int32)), int(counts.sum())
    before, slots = lens.clone(), torch.empty(total, dtype=torch.int64, device="cuda")
    batch_ = r.batch()
    tm.tm_paged_assign(r.cache, r.list, batch_, lens, counts, slots=slots)
    assert torch.equal(lens, before + counts) and int(r.list.count) == 4
    valid = slots[slots >= 0]
    assert valid.numel() == total and valid.unique().numel() == total      # every token has a slot of its own
    table, first = r.T.clone(), slots.clone()
    tm.tm_paged_release(r.cache, r.list, r.T, first=before)
    assert np.array_equal(_host(r.T), r.table) and np.array_equal(_host(r.list.pages), r.pages) and int(r.list.count) == r.count
    lens.copy_(before)
    tm.tm_paged_assign(r.cache, r.list, batch_, lens, counts, slots=slots)
    assert torch.equal(r.T, table) and torch.equal(slots, first)


@pytest.mark.parametrize("batch", [40, 1100, 5000])
def test_captured_steps_go_on(tm, batch):
    """A captured step that updates lengths and list in place, replayed: every replay goes on where the last one ended.  Eager work between the replays."""
    import torch
    r = Rows(tm, [i % 70 for i in range(batch)], 32, 8, 6 * batch)
    lens, counts = _dev(r.lens), torch.ones(batch, dtype=torch.int32, device="cuda")
    slots, batch_ = torch.empty(4 * batch, dtype=torch.int64, device="cuda"), r.batch()
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(g, stream=side):
        tm.tm_paged_assign(r.cache, r.list, batch_, lens, counts, slots=slots)
    table, count, n = r.table, r.count, r.lens
    for step in range(4):
        counts.fill_(step)
        want = st.assign(r.pages.tolist(), count, n, [step] * batch, table, 32, r.pool, 4 * batch)
        g.replay()
        torch.cuda.synchronize()
        table, count, n = want["table"], want["left"], want["lens"]
        assert np.array_equal(_host(r.T), table) and int(r.list.count) == count and np.array_equal(_host(lens), n)
        assert _host(slots)[:step * batch].tolist() == [want["slots"][t] for t in range(step * batch)]
        _ = (torch.randn(1000, 1000, device="cuda") @ torch.randn(1000, 1000, device="cuda")).sum().item()


def test_refusals(tm):
    import torch
    r = Rows(tm, [1, 2], 32, 4, 4)
    ints = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    b, both = r.batch(), ints(4, 2)
    for call, error, text in [
            (lambda: tm.tm_paged_assign(r.cache, r.list, b, ints(2), ints(2)), ValueError, "slots or tokens"),
            (lambda: tm.tm_paged_assign(r.cache, r.list, b, ints(3), ints(2), tokens=4), ValueError, "lens"),
            (lambda: tm.tm_paged_assign(r.cache, r.list, b, ints(2), ints(1), tokens=4), ValueError, "counts"),
            (lambda: tm.tm_paged_assign(r.cache, r.list, b, ints(2), ints(2), slots=ints(4)), TypeError, "int64"),
            (lambda: tm.tm_paged_assign(r.cache, r.list, b, ints(2), ints(2), slots=torch.zeros(3, dtype=torch.int64, device="cuda"), tokens=4), ValueError, "slots"),
            (lambda: tm.tm_paged_assign(r.cache, r.list, b, b.positions, ints(2), tokens=4), tm.TmError, "overlap"),
            (lambda: tm.tm_paged_assign(r.cache, r.list, b, ints(2), b.positions, tokens=4), tm.TmError, "overlap"),
            (lambda: tm.tm_paged_assign(r.cache, r.list, b, both[0], both[0], tokens=4), tm.TmError, "lens_out .* counts"),
            (lambda: tm.tm_paged_assign(r.cache, r.list, b, both[:2].reshape(-1)[:2], ints(2), lens_out=both.reshape(-1)[1:3], tokens=4), tm.TmError, "lens_out .* lens"),
            (lambda: tm.tm_paged_assign(r.cache, r.list, b, ints(2), ints(2), left=b.offsets[:1], tokens=4), tm.TmError, "left .* offsets"),
            (lambda: tm.tm_paged_assign(r.cache, tm.PageList(r.list.pages, r.list.pages[:1]), b, ints(2), ints(2), tokens=4), tm.TmError, "left .* pages"),
            (lambda: tm.tm_paged_assign(r.cache, r.list, b, ints(2), ints(2), short=r.T.reshape(-1)[3:5], tokens=4), tm.TmError, "table .* lacking"),
            (lambda: tm.tm_paged_release(r.cache, r.list, r.T, first=r.T.reshape(-1)[2:4]), tm.TmError, "table .* from"),
            (lambda: tm.tm_paged_release(r.cache, tm.PageList(r.T.reshape(-1), r.list.count), r.T), tm.TmError, "pages .* table"),
            (lambda: tm.tm_paged_assign(r.cache, tm.PageList(ints(4), ints(2)), b, ints(2), ints(2), tokens=4), ValueError, "count"),
            (lambda: tm.tm_paged_assign(r.cache, r.list, b, ints(2).cpu(), ints(2), tokens=4), TypeError, "device"),
            (lambda: tm.tm_paged_release(r.cache, r.list, ints(8)), ValueError, "table"),
            (lambda: tm.tm_paged_release(r.cache, r.list, r.T, first=ints(3)), ValueError, "first")]:
        with pytest.raises(error, match=text):
            call()
