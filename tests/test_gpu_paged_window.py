"""GPU parity of attention in a sliding window over a paged cache (tm_paged_attn_window) against the 64-bit oracle.  Set-up and tolerance are those of the full attention's tests
(test_gpu_paged_attn.py): one rounding of the result, one of every probability times its value's scale, an eighth of both for what fp32 sums add to scores and probabilities.

The value sums need a term of their own here: that eighth is taken of A, the average of |V^|, and a window of a few tokens may have values that are all zero in a dimension (A = 0), where what
is left is the fp32 error of the sums of codes.  A code goes in with the conversion's bias, at most 1024 + 15 units of the value's scale (4-bit) or 1024 + 127 (8-bit, centred), and the bias
leaves again.  With S, the average of the scales, a sum never exceeds 1039 S (1151 S).  One rounding is 2^-24 of the sum so far.  A matrix instruction adds 32 products in at most
eight steps; over a block the sum goes up from zero evenly, so its steps are worth 1/8 + 2/8 + ... + 1 = 4.5 roundings of the block's largest sum; the bias is summed up alike (4.5) and added
(1).  4-bit codes: 10 roundings of each block's share of 1039 S, together 10 * 2^-24 * 1039 S.  8-bit codes: the bias leaves every fourth block, so sums reach four blocks' share, in
2.5 on average: 25 * 2^-24 * 1151 S."""
import sys

import numpy as np
import pytest

from oracle import oracle_paged as op
from oracle import oracle_step as st
from test_gpu_paged_attn import SCALE, Setup, _dev, _host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tm():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_2508_15601_amd as tm
    tm.load_library()
    return tm


class Window(Setup):
    """Pages that no new token of a sequence sees are given to others: -1, or a page of arbitrary bytes."""

    def __init__(self, tm, window, sinks, *args, taken=True, **kw):
        super().__init__(tm, *args, **kw)
        self.window, self.sinks = window, sinks
        if taken:
            for b, (n, p) in enumerate(zip(self.counts, self.positions)):
                lo = max(p, 0) - window + 1
                for c in range(self.table.shape[1]):
                    if n and c * self.page >= sinks and (c + 1) * self.page <= lo:
                        self.table[b, c] = [-1, self.k.shape[0] - 1, self.k.shape[0] + 5][c % 3]
            self.batch.table.copy_(_dev(self.table))

    def run(self):
        import torch
        O = torch.full_like(self.Q, 7.0)
        self.tm.tm_paged_attn(self.Q, self.cache, self.batch, O, SCALE, window=self.window, sinks=self.sinks)
        return O

    def want(self):
        arrays = op.unpack_pool(_host(self.k), _host(self.v), _host(self.pairs))
        return st.attention(_host(self.Q), arrays, self.table, self.offsets, self.positions, SCALE, self.window, self.sinks)

    def check(self):
        import torch
        print(f"bits={self.bits} page={self.page} heads={self.q_heads}/{self.heads} window={self.window} sinks={self.sinks} counts={self.counts[:6]} positions={self.positions[:6]} "
              f"plan={self.plan()}", file=sys.stderr, flush=True)
        O = self.run()
        got = _host(O).astype(np.float64)
        want, A, S = self.want()
        untouched = np.isnan(want)
        assert (got[untouched] == 7).all()
        g, w, a, s = (x[~untouched] for x in (got, want, A, S))
        assert np.isfinite(g).all()
        sums = 2.0 ** -24 * (10 * 1039 if self.bits == 4 else 25 * 1151) * s
        worst = (np.abs(g - w) / (1.125 * 2.0 ** -11 * (np.abs(w) + a) + 2.0 ** -25 + sums)).max() if g.size else 0.0
        assert worst <= 1.0, worst
        assert torch.equal(self.run(), O)                                  # bit-identical from run to run: the workspace was left ready


FEW = [
    # window, sinks, page, KV heads, query heads, counts, positions
    (1, 0, 32, 1, 1, [1], [0]),
    (1, 0, 32, 2, 8, [1, 1, 1], [1, 31, 700]),                             # a token's own value
    (5, 1, 32, 2, 8, [1, 1, 1, 1], [0, 3, 64, 900]),
    (32, 4, 64, 2, 10, [1, 1, 1, 1], [127, 128, 700, 63]),
    (33, 0, 32, 1, 16, [1, 1], [500, 99]),
    (100, 33, 128, 1, 40, [1, 1], [300, 17]),                              # more query heads than columns
    (64, 64, 64, 1, 64, [1], [1000]),                                      # whole blocks, nothing at their edges
    (128, 200, 256, 2, 14, [2, 0, 4, 1], [1000, 5, 254, 0]),               # more first tokens than window
    (40, 2, 32, 3, 3, [8, 3], [90, 0]),                                    # tokens of a sequence with windows of their own
    (3, 0, 1024, 1, 5, [5, 5], [1500, 1]),
    (50, 10, 64, 2, 8, [16, 13], [200, 64]),                               # column tiles
    (7, 130, 32, 1, 4, [12], [500]),
    (300, 3, 32, 1, 8, [1, 1], [-1, -400]),                                # no positions at all
    (5000, 1, 64, 2, 8, [1, 2], [700, 20]),                                # the window is longer than everything
]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("window, sinks, page, heads, q_heads, counts, positions", FEW)
def test_few_tokens(tm, bits, window, sinks, page, heads, q_heads, counts, positions):
    Window(tm, window, sinks, bits, page, heads, counts, positions, q_heads=q_heads, before=1, behind=2, max_count=max(counts), seed=q_heads).check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("heads, q_heads, context, window, sinks", [(1, 4, 9000, 6000, 4), (1, 16, 6000, 3000, 0), (4, 4, 30000, 1000, 70), (2, 16, 20000, 15000, 129),
                                                                     (1, 1, 70000, 50000, 1)])
def test_one_long_context(tm, bits, heads, q_heads, context, window, sinks):
    """Cut into pieces: in one level and in two, the gap inside a piece."""
    Window(tm, window, sinks, bits, 64, heads, [1], [context - 1], q_heads=q_heads, max_count=1, seed=context).check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("batch, window, sinks", [(5, 500, 4), (64, 100, 0), (65, 1000, 40), (200, 64, 4), (1100, 200, 5)])
def test_contexts_of_very_different_lengths(tm, bits, batch, window, sinks):
    """The last one with a wave to a segment, in either width of codes."""
    rng = np.random.default_rng(batch)
    positions = (3000 * rng.random(batch) ** 6).astype(int)
    positions[batch // 2] = 5000
    counts = rng.choice([0, 1, 1, 1], batch)
    counts[batch // 2] = 1
    if batch > 1000:
        positions = np.minimum(positions, 900)
    s = Window(tm, window, sinks, bits, 32, 1 if batch > 64 else 2, counts.tolist(), positions.tolist(), q_heads=4, max_count=1, max_len=5001, seed=batch)
    if batch > 1000:
        assert tm.tm_get_paged_form(s.cache, s.batch, s.tokens, s.q_heads)[2]
    s.check()


MANY = [
    # window, sinks, page, KV heads, query heads, counts, positions
    (50, 4, 32, 1, 1, [300, 77], [0, 500]),
    (1, 0, 64, 1, 4, [200], [33]),
    (64, 64, 64, 2, 8, [130], [640]),
    (200, 3, 64, 1, 8, [100, 1, 300], [1000, 900, 0]),                     # decoding sequences beside chunks
    (1000, 0, 128, 1, 4, [500], [4000]),
    (129, 300, 32, 1, 7, [90, 17, 2], [700, 100, 350]),                    # more first tokens than window
    (31, 1, 256, 2, 32, [40, 9], [900, 1200]),
    (70, 5, 32, 1, 5, [400], [-60]),                                       # begins before the first position
    (90, 0, 32, 1, 64, [33], [400]),                                       # a token's rows over more than one tile
    (2000, 40, 64, 1, 8, [600], [0]),
]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("window, sinks, page, heads, q_heads, counts, positions", MANY)
def test_many_tokens(tm, bits, window, sinks, page, heads, q_heads, counts, positions):
    s = Window(tm, window, sinks, bits, page, heads, counts, positions, q_heads=q_heads, before=2, behind=1, max_count=max(counts), seed=window)
    assert s.plan()[2], s.plan()
    s.check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("hints", [{}, dict(max_count=64), dict(max_count=700, max_len=3000)])
def test_hints_do_not_matter(tm, bits, hints):
    Window(tm, 150, 20, bits, 64, 1, [64, 1, 30], [2500, 300, 0], q_heads=8, seed=1, **hints).check()


@pytest.mark.parametrize("bits", [8, 4])
def test_a_chunk_in_pieces(tm, bits):
    """Few row tiles and a long window: contexts in pieces, with 128 and 256 rows a CTA."""
    for counts, q_heads, window in ([70], 4, 9000), ([17], 64, 5000), ([300], 4, 7000):
        s = Window(tm, window, 100, bits, 64, 1, counts, [12000], q_heads=q_heads, max_count=counts[0], max_len=12000 + counts[0], seed=counts[0])
        assert s.plan()[2] and s.plan()[3] > 1, s.plan()
        s.check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("counts, positions", [([1, 1, 1], [500, 300, 77]), ([90, 1, 200], [500, 300, 77])])
def test_pages_missing_inside_the_window(tm, bits, counts, positions):
    """Tokens on pages that the pool does not have are not seen; a row that is left with none is zero."""
    bad = [(0, c, -1) for c in range(12, 18)] + [(1, c, 1 << 20) for c in range(0, 10)] + [(2, 2, -5)]
    s = Window(tm, 40, 0, bits, 32, 2, counts, positions, q_heads=8, bad=bad, cols=32, seed=5, taken=False)
    s.check()
    O = _host(s.run())
    assert (O[s.offsets[1]] == 0).all() and (O[0] == 0).all() and (O[s.offsets[2]] != 0).any()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("counts, positions, q_heads", [([1, 1], [900, 30], 8), ([5, 2], [900, 30], 8), ([100, 3], [900, 30], 8)])
def test_a_window_over_everything_is_full_attention(tm, bits, counts, positions, q_heads):
    """Bit for bit where the window and the first tokens reach as far as the table; the same to rounding where they only reach as far as the sequences."""
    import torch
    s = Window(tm, 1, 0, bits, 64, 2, counts, positions, q_heads=q_heads, seed=2, taken=False)
    full = torch.empty_like(s.Q)
    tm.tm_paged_attn(s.Q, s.cache, s.batch, full, SCALE)
    for window, sinks in ((s.cap, 0), (1 << 30, 0), ((1 << 31) - 1, (1 << 31) - 1), (1, s.cap), (s.cap - 8, 8)):
        s.window, s.sinks = window, sinks
        assert torch.equal(s.run(), full), (window, sinks)
    s.window, s.sinks = 1000, 3
    s.check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("counts, positions, q_heads, max_count", [([1, 1], [900, 300], 8, 1), ([5, 2], [900, 30], 32, 0), ([100, 3], [900, 30], 8, 100)])
def test_offsets_past_32_bits(tm, bits, counts, positions, q_heads, max_count):
    """Pages whose codes lie beyond 2^32 bytes, stored with norms and positions of their own: as on the pool's first pages, bit for bit, and nothing between them is written."""
    import torch
    page, heads, cols = 256, 8, 4
    pages = 17000 if bits == 8 else 34000                                  # 4.4 GB of key codes
    k, v, pairs = tm.tm_paged_pool(pages, heads, page, bits)
    cache = tm.tm_paged_create(k, v, pairs)
    total = sum(counts)
    offsets = _dev(np.array([0, counts[0], total], np.int32))
    g = torch.Generator(device="cuda").manual_seed(bits + total)
    K, V, Q = (torch.randn(n, h, 128, generator=g, device="cuda").half() for n, h in ((1000, heads), (1000, heads), (total, q_heads)))
    rope, norm = tm.tm_rope_create(128, axis=[i % 2 for i in range(64)]), tm.HeadNorm(K[0, 0].clone())
    at = torch.randint(0, 5000, (1000, 2), generator=g, device="cuda", dtype=torch.int32)
    out = []
    for ids in (np.arange(2 * cols), np.arange(pages - 2 * cols, pages)):
        table = _dev(ids.reshape(2, cols).astype(np.int32))
        for b in range(2):                                                 # what the new tokens see of their sequences
            n = positions[b] + counts[b]
            tm.tm_paged_append(cache, tm.PagedBatch(table[b:b + 1].contiguous(), _dev(np.array([0, n], np.int32)), _dev(np.zeros(1, np.int32))), K[:n], V[:n], rope=rope, k_norm=norm,
                               positions=at[:n])
        O = torch.empty_like(Q)
        batch = tm.PagedBatch(table, offsets, _dev(np.array(positions, np.int32)), max_count=max_count)
        out.append((tm.tm_paged_attn(Q, cache, batch, O, SCALE, window=200, sinks=5), [x[torch.as_tensor(ids, device="cuda")] for x in (k, v, pairs)]))
    assert torch.equal(out[0][0], out[1][0]) and out[0][0].isfinite().all() and out[0][0].any()
    assert all(torch.equal(x, y) for x, y in zip(out[0][1], out[1][1]))
    assert not pairs[2 * cols:-2 * cols].any() and not k[2 * cols:-2 * cols].any()


def test_in_a_graph(tm):
    """Captured, and replayed with tables, positions and queries that changed in between; two graphs over one workspace in turn."""
    import torch
    few = Window(tm, 100, 4, 8, 64, 2, [1] * 9, [60 * i for i in range(9)], q_heads=8, max_count=1, max_len=600, cols=10, seed=3, taken=False)
    many = Window(tm, 100, 4, 4, 64, 2, [100, 1], [700, 900], q_heads=8, max_count=100, cols=20, seed=4, taken=False)
    many.cache.close()
    many.cache = tm.tm_paged_create(many.k, many.v, many.pairs, few.cache.workspace)
    out, graphs = [], []
    for s in (few, many):
        O, g = torch.zeros_like(s.Q), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            tm.tm_paged_attn(s.Q, s.cache, s.batch, O, SCALE, window=s.window, sinks=s.sinks)
        out.append(O)
        graphs.append(g)
    for step in range(4):
        for s, O, g in zip((few, many), out, graphs):
            s.Q.mul_(0.9)
            s.batch.positions.add_(3)
            O.fill_(7)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(s.run().view(torch.int16), O.view(torch.int16))    # (the tokens the positions moved on to hold arbitrary bytes, NaN among them)
            _ = (torch.randn(1000, 1000, device="cuda") @ torch.randn(1000, 1000, device="cuda")).sum().item()


def test_refusals(tm):
    s = Window(tm, 10, 0, 8, 32, 1, [1], [5], q_heads=4)
    for window, sinks, error in ((0, 0, tm.TmError), (-1, 0, tm.TmError), (5, -1, tm.TmError), (None, 4, ValueError), (1 << 31, 0, ValueError), (1, 1 << 40, ValueError)):
        with pytest.raises(error):
            tm.tm_paged_attn(s.Q, s.cache, s.batch, s.Q.clone(), SCALE, window=window, sinks=sinks)
