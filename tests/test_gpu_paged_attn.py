"""GPU parity of attention over a paged cache (tm_paged_attn) against the 64-bit oracle.

Tolerance, per value: the result is rounded to fp16 once (2^-11 of it) and every probability times value scale once (2^-11 of its term, so 2^-11 of A = sum p |V^| at
most).  What is summed in fp32 comes on top: scores carry the bias of the code conversion, up to 1279 times the sum of |q| against the codes' own 255, which moves an exponent by less than
1e-4 here, and so a probability; the value sums likewise, 1151 (4-bit: 1039) units against up to 127 (7) and 2^-24 a step.  An eighth of the two roundings covers both."""
import sys

import numpy as np
import pytest

from oracle import oracle_paged as op

pytestmark = pytest.mark.gpu

SCALE = 128 ** -0.5


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


class Setup:
    """A pool of arbitrary bytes (NaN and infinite scales among them) in which the sequences' tokens have been stored, and nothing else."""

    def __init__(self, tm, bits, page, heads, counts, positions, cols=None, seed=0, before=0, behind=0, q_heads=None, bad=(), spread=1.0, **hints):
        import torch
        rng = np.random.default_rng(seed)
        B = len(counts)
        last = [max(0, p + n) for p, n in zip(positions, counts)]
        cols = cols or max(1, max(-(-n // page) for n in last))
        self.tm, self.bits, self.page, self.heads, self.cap = tm, bits, page, heads, cols * page
        last = [min(n, self.cap) for n in last]
        pages = B * cols + 2
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.k, self.v = (torch.randint(0, 256, (pages, heads, page // 32, 512 * bits), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
        self.pairs = torch.randint(-32768, 32768, (pages, heads, page, 2, 2), generator=g, device="cuda", dtype=torch.int16).view(torch.float16)
        self.table = rng.permutation(pages)[:B * cols].reshape(B, cols).astype(np.int32)
        self.offsets = (before + np.cumsum([0] + list(counts))).astype(np.int32)
        self.counts, self.positions = counts, list(positions)
        self.tokens = int(self.offsets[-1]) + behind
        self.cache = tm.tm_paged_create(self.k, self.v, self.pairs)
        # everything up to the sequences' ends
        fill = tm.PagedBatch(_dev(self.table), _dev(np.cumsum([0] + last).astype(np.int32)), torch.zeros(B, dtype=torch.int32, device="cuda"))
        K, V = (torch.randn(sum(last), heads, 128, generator=g, device="cuda").mul_(spread).half() for _ in range(2))
        tm.tm_paged_append(self.cache, fill, K, V)
        for b, c, value in bad:
            self.table[b, c] = value
        self.batch = tm.PagedBatch(_dev(self.table), _dev(self.offsets), _dev(np.asarray(positions, np.int32)), **hints)
        self.q_heads = q_heads or heads
        self.Q = torch.randn(self.tokens, self.q_heads, 128, generator=g, device="cuda").half()

    def plan(self):
        return self.tm.tm_get_paged_plan(self.cache, self.batch, self.tokens, self.q_heads)

    def run(self):
        import torch
        O = torch.full_like(self.Q, 7.0)
        self.tm.tm_paged_attn(self.Q, self.cache, self.batch, O, SCALE)
        return O

    def want(self):
        arrays = op.unpack_pool(_host(self.k), _host(self.v), _host(self.pairs))
        return op.attention(_host(self.Q), arrays, self.table, self.offsets, self.positions, SCALE)

    def check(self, form=None):
        import torch
        plan = self.plan()
        print(f"bits={self.bits} page={self.page} heads={self.q_heads}/{self.heads} counts={self.counts[:6]} positions={self.positions[:6]} plan={plan}", file=sys.stderr, flush=True)
        if form is not None:
            assert tuple(x > 0 if isinstance(f, bool) else x for x, f in zip(plan, form)) == form, plan
        O = self.run()
        got = _host(O).astype(np.float64)
        want, A = self.want()
        untouched = np.isnan(want)
        assert (got[untouched] == 7).all()
        g, w, a = got[~untouched], want[~untouched], A[~untouched]
        assert np.isfinite(g).all()
        worst = (np.abs(g - w) / (1.125 * 2.0 ** -11 * (np.abs(w) + a) + 2.0 ** -25)).max() if g.size else 0.0
        assert worst <= 1.0, worst
        assert torch.equal(self.run(), O)                                  # bit-identical from run to run: the workspace was left ready
        return O


# form: (columns, column_rows, rows, pieces) of the plan; True / False: more than 0 / 0
FEW = [
    # page, KV heads, query heads, counts, positions, columns
    (32, 1, 1, [1], [0], 8),                                               # one token, one head
    (32, 2, 8, [1, 1, 1], [0, 31, 32], 8),                                 # last slot of a page, first of the next
    (64, 2, 10, [1, 1, 1, 1], [127, 128, 700, 63], 8),                     # blocks of 8- and 4-bit codes that end inside a page
    (32, 1, 16, [1, 1], [500, 99], 16),
    (128, 1, 40, [1, 1], [300, 17], 32),                                   # more query heads than columns
    (64, 1, 64, [1], [1000], 32),
    (256, 2, 14, [2, 0, 4, 1], [1000, 5, 254, 0], 32),                     # drafted tokens; a sequence without any
    (32, 3, 3, [8, 3], [90, 0], 8),
    (1024, 1, 5, [5, 5], [1500, 1], 32),
    (64, 2, 8, [16, 13], [200, 64], 32),                                   # several column tiles of a sequence
]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("page, heads, q_heads, counts, positions, columns", FEW)
def test_few_tokens(tm, bits, page, heads, q_heads, counts, positions, columns):
    s = Setup(tm, bits, page, heads, counts, positions, q_heads=q_heads, before=1, behind=2, max_count=max(counts), seed=q_heads)
    s.check((columns, True, 0, 0))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("heads, q_heads, context", [(1, 4, 9000), (1, 16, 6000), (4, 4, 3333), (2, 16, 20000), (1, 1, 70000)])
def test_one_long_context(tm, bits, heads, q_heads, context):
    """Cut into many pieces: in one level and in two."""
    Setup(tm, bits, 64, heads, [1], [context - 1], q_heads=q_heads, max_count=1, seed=context).check((8 if q_heads // heads <= 8 else 16, True, 0, 0))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("batch", [5, 64, 65, 200])
def test_contexts_of_very_different_lengths(tm, bits, batch):
    rng = np.random.default_rng(batch)
    positions = (3000 * rng.random(batch) ** 6).astype(int)
    positions[batch // 2] = 5000
    counts = rng.choice([0, 1, 1, 1], batch)
    counts[batch // 2] = 1
    Setup(tm, bits, 32, 1 if batch > 64 else 2, counts.tolist(), positions.tolist(), q_heads=4, max_count=1, max_len=5001, seed=batch).check((8, True, 0, 0))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("counts, positions", [([1] * 6, [0, 900, 31, 32, 300, 64]), ([0] * 20 + [19], [100 + i for i in range(20)] + [400])])
def test_no_hints_and_no_more_tokens_than_sequences(tm, bits, counts, positions):
    """Taken for a decoding step; right where it is none."""
    Setup(tm, bits, 64, 2, counts, positions, q_heads=8, before=0, behind=0, seed=len(counts)).check((8, True, 0, 0))


def _lengths(batch, longest, seed):
    rng = np.random.default_rng(seed)
    lengths = (40 + 200 * rng.random(batch)).astype(int)
    lengths[batch // 3] = longest
    return lengths.tolist()


@pytest.mark.parametrize("page, heads, q_heads, batch, longest, count, columns", [
    (32, 8, 32, 40, 700, 1, 8),                                            # a few segments more than compute units: pieces of a segment
    (64, 8, 8, 40, 3600, 1, 8),                                            # one sequence in more than sixteen pieces
    (64, 4, 48, 70, 300, 1, 16),                                           # more sequences than lanes
    (128, 8, 40, 34, 500, 5, 16),                                          # more columns than a tile
    (32, 2, 6, 131, 400, 2, 8),
])
def test_many_segments_4bit(tm, page, heads, q_heads, batch, longest, count, columns):
    """More segments than compute units: every wave works by itself."""
    counts = [count] * batch
    counts[1] = 0
    Setup(tm, 4, page, heads, counts, _lengths(batch, longest, page), q_heads=q_heads, before=1, behind=1, max_count=count, seed=batch).check((columns, True, 0, 0))


@pytest.mark.parametrize("page, heads, q_heads, batch, longest, count, max_len, columns", [
    (64, 16, 32, 64, 1500, 1, 1501, 8),
    (32, 16, 160, 66, 300, 1, 0, 16),
    (64, 16, 32, 64, 200, 3, 0, 8),
    (64, 8, 32, 33, 500, 1, 501, 8),                                       # short contexts: two CTAs a compute unit
    (32, 4, 40, 90, 700, 1, 701, 16),
])
def test_many_segments_8bit(tm, page, heads, q_heads, batch, longest, count, max_len, columns):
    counts = [count] * batch
    counts[1] = 0
    Setup(tm, 8, page, heads, counts, _lengths(batch, longest, page), q_heads=q_heads, before=1, behind=1, max_count=count, max_len=max_len, seed=batch).check((columns, True, 0, 0))


@pytest.mark.parametrize("bits", [8, 4])
def test_many_segments_and_bad_pages(tm, bits):
    """Sequences of missing pages only, first, in the middle and last, and with lengths of none: every wave by itself."""
    batch = 130 if bits == 8 else 40
    lengths = _lengths(batch, 333, 5)
    bad = [(3, c, -1) for c in range(11)] + [(5, 0, 1 << 30), (7, 1, -2), (9, lengths[9] // 32, -5)]
    positions = list(lengths)
    positions[11], positions[12] = -1, -4
    Setup(tm, bits, 32, 8, [1] * batch, positions, q_heads=16, max_count=1, seed=3, bad=bad).check((8, True, 0, 0))


def test_work_of_a_wide_table_is_counted_in_32_bits(tm):
    """Every wave by itself counts its work in blocks, four to a CTA's unit: not where a table is so wide that the count might not fit."""
    import torch
    k, v, pairs = tm.tm_paged_pool(2, 8, 64, 4)
    cache = tm.tm_paged_create(k, v, pairs)
    offsets, positions = torch.arange(0, 175, 5, dtype=torch.int32, device="cuda"), torch.zeros(34, dtype=torch.int32, device="cuda")
    for cols, columns in ((1 << 20, 16), (1 << 21, 32)):
        table = torch.zeros(34, cols, dtype=torch.int32, device="cuda")
        assert tm.tm_get_paged_plan(cache, tm.PagedBatch(table, offsets, positions, max_count=5), 170, 32)[0] == columns


MANY = [
    # page, KV heads, query heads, counts, positions
    (64, 1, 4, [65], [0]),                                                 # a whole prompt
    (32, 2, 8, [70], [1000]),                                              # a chunk after a long past: pieces
    (128, 1, 7, [150], [33]),
    (32, 1, 1, [300], [45]),
    (256, 1, 16, [40, 31], [300, 0]),
    (64, 2, 2, [129, 200, 77], [0, 100, 1000]),                            # packed prompts of different lengths
    (64, 8, 8, [400], [0]),
]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("page, heads, q_heads, counts, positions", MANY)
def test_many_tokens(tm, bits, page, heads, q_heads, counts, positions):
    Setup(tm, bits, page, heads, counts, positions, q_heads=q_heads, before=3, behind=2, seed=sum(counts)).check((len(counts) > 1, len(counts) > 1, True, True))


@pytest.mark.parametrize("bits", [8, 4])
def test_pieces_of_a_chunk(tm, bits):
    """The pieces of a context end inside and at the end of pages, and the last one is short."""
    for past in (2000, 4095, 4096 - 70):
        s = Setup(tm, bits, 32, 1, [70], [past], q_heads=4, seed=past)
        assert s.plan()[3] > 4
        s.check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("counts, positions, heads, q_heads", [
    ([300, 90, 200], [4000, 2500, 100], 1, 4),                             # cut into different numbers of pieces, one into none
    ([1] * 40 + [70] + [1] * 40 + [33, 150], [50 * i for i in range(40)] + [3000] + [9 * i for i in range(40)] + [1200, 0], 1, 8),   # more sequences than lanes
    ([64, 0, 64, 2], [6000, 100, 5900, 3000], 2, 4),
])
def test_pieces_of_several_chunks(tm, bits, counts, positions, heads, q_heads):
    s = Setup(tm, bits, 64, heads, counts, positions, q_heads=q_heads, before=2, behind=1, seed=len(counts), max_count=max(counts))
    assert s.plan()[3] > 4
    s.check()


@pytest.mark.parametrize("bits", [8, 4])
def test_mixed(tm, bits):
    """Decoding sequences, drafts, chunks and prompts in one call."""
    counts = [1, 1, 90, 1, 0, 5, 1, 33, 1, 170, 1, 2]
    positions = [700, 0, 31, 64, 9, 1500, 32, 0, 2000, 300, 5, 63]
    Setup(tm, bits, 64, 2, counts, positions, q_heads=8, before=4, behind=1, seed=1).check((True, True, True, True))
    Setup(tm, bits, 32, 1, counts, positions, q_heads=12, seed=2, max_count=170, max_len=2001).check((True, True, True, True))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("page, heads, q_heads, counts, positions", [
    (32, 2, 24, [1, 40, 1, 1, 9, 1], [300, 500, 0, 95, 64, 2100]),         # sixteen columns; parts of a block on pages of their own
    (32, 1, 3, [2, 200, 5, 1], [33, 3000, 700, 4000]),
    (128, 8, 8, [1] * 70 + [300], [11 * i for i in range(70)] + [50]),     # more sequences than lanes, and more segments than waves
])
def test_mixed_forms(tm, bits, page, heads, q_heads, counts, positions):
    Setup(tm, bits, page, heads, counts, positions, q_heads=q_heads, before=1, behind=2, seed=page, max_count=max(counts), max_len=max(n + p for n, p in zip(counts, positions))).check(
        (True, True, True, True))


def test_mixed_over_a_wide_table(tm):
    """Wider than a wave's count of blocks allows: two launches."""
    s = Setup(tm, 8, 64, 8, [1, 100, 3], [200, 900, 70], q_heads=32, seed=5, max_count=100, max_len=1000)
    s.check((True, True, True, True))
    s.table = np.pad(s.table, ((0, 0), (0, 2600000 - s.table.shape[1])), constant_values=-1)
    s.batch = tm.PagedBatch(_dev(s.table), s.batch.offsets, s.batch.positions, max_count=100, max_len=1000)
    s.check((True, True, True, True))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("hints", [dict(), dict(max_count=1), dict(max_count=1, max_len=1), dict(max_count=5, max_len=10), dict(max_len=40), dict(max_count=1 << 20, max_len=1 << 20)])
def test_results_do_not_depend_on_the_hints(tm, bits, hints):
    """Hints that are missing, far too small or too large."""
    Setup(tm, bits, 32, 1, [1, 60, 7, 1, 150], [900, 100, 0, 5, 333], q_heads=4, seed=3, **hints).check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("counts, positions", [([1, 1, 1], [200, 100, 95]), ([3, 80, 100], [200, 100, 0])])
def test_pages_that_do_not_exist(tm, bits, counts, positions):
    """Holes in a context, at its beginning and end; a sequence with no page at all."""
    bad = [(0, 1, -1), (0, 3, 1 << 30), (1, 0, -5), (1, 4, -1), (2, 0, -1), (2, 1, -1), (2, 2, -1), (2, 3, -1), (2, 4, -1), (2, 5, -1)]
    s = Setup(tm, bits, 32, 2, counts, positions, cols=8, q_heads=8, bad=bad, seed=4)
    O = s.check()
    assert (_host(O)[s.offsets[2]:s.offsets[3]] == 0).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_positions_outside_the_table(tm, bits):
    """Rows before the first slot and behind the last are left as they were."""
    Setup(tm, bits, 32, 1, [4, 3, 2, 1], [-2, 62, 64, -1], cols=2, q_heads=4, before=1, seed=5).check()
    Setup(tm, bits, 32, 1, [100, 90, 70], [-50, 60, 128], cols=4, q_heads=2, seed=6).check()
    Setup(tm, bits, 32, 1, [1, 1], [2 ** 31 - 1, -2 ** 31], cols=2, q_heads=2, seed=7).check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("counts, positions", [([1, 1], [600, 40]), ([100], [200])])
def test_scores_of_any_size(tm, bits, counts, positions):
    """Keys fifty times as large: one token takes nearly all of the probability, and the fp32 errors of a score are no longer small.  The column form multiplies q with codes that
    carry a bias, at most 1279 in all, and takes it out again: 4 x 4 steps of a matrix product and 34 additions for the bias, each rounding sums of up to 1279 sum |q| by
    2^-24.  Times the key's scale and the softmax scale that is the exponent's error d; probabilities are off by a factor of e^(+-d) each, a quotient of their sums by e^(+-2d).
    The value sums carry a bias as well, and where V^ is 0 nothing else is left: 3 or 5 blocks a wave with 4 or 3 additions each and 8 to join the waves, at most 24, each rounding
    a sum of up to 1279 times the sum of probability times value scale by 2^-24."""
    s = Setup(tm, bits, 32, 1, counts, positions, q_heads=4, spread=50.0, seed=8)
    O = _host(s.run()).astype(np.float64)
    want, A = s.want()
    Q = np.abs(_host(s.Q).astype(np.float64)).sum(-1)
    arrays = op.unpack_pool(_host(s.k), _host(s.v), _host(s.pairs))
    for b, (n, p) in enumerate(zip(counts, positions)):
        rows = slice(s.offsets[b], s.offsets[b + 1])
        t = np.arange(p + n)
        scale = arrays[1][s.table[b, t // s.page], 0, t % s.page].astype(np.float64).max()
        values = arrays[4][s.table[b, t // s.page], 0, t % s.page].astype(np.float64).max()
        d = 50 * 2.0 ** -24 * 1279 * Q[rows] * scale * SCALE
        bound = 1.125 * 2.0 ** -11 * (np.abs(want[rows]) + A[rows]) + np.expm1(2 * d)[..., None] * 2 * A[rows] + 24 * 2.0 ** -24 * 1279 * values + 2.0 ** -25
        assert (np.abs(O[rows] - want[rows]) <= bound).all()


def test_rows_apart_and_another_stream(tm):
    import torch
    s = Setup(tm, 8, 64, 2, [1, 40, 1], [100, 50, 0], q_heads=4, seed=9)
    want = s.run()
    qkv = torch.full((s.tokens, 8, 128), float("nan"), dtype=torch.float16, device="cuda")
    qkv[:, :4] = s.Q
    O = torch.empty_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    tm.tm_paged_attn(qkv[:, :4], s.cache, s.batch, O, SCALE, stream=side)
    side.synchronize()
    assert torch.equal(O, want)


@pytest.mark.parametrize("bits", [8, 4])
def test_steps_in_a_graph(tm, bits):
    """A serving step - rotate and store, attend - captured once and replayed for the following tokens, against eager calls on a copy of the pool; the workspace is
    shared by two layers and with eager calls in between."""
    import torch
    counts, q_heads, heads = [1, 70, 3], 8, 2
    a = Setup(tm, bits, 32, heads, counts, [900, 100, 30], cols=40, q_heads=q_heads, seed=10)
    b = Setup(tm, bits, 32, heads, counts, [900, 100, 30], cols=40, q_heads=q_heads, seed=10)
    ws = tm.tm_paged_workspace()
    layers = [(tm.tm_paged_create(s.k, s.v, s.pairs, ws), s) for s in (a, b)]
    rope = tm.tm_rope_create(128)
    qkv = torch.randn(2, a.tokens, q_heads + 2 * heads, 128, device="cuda").half()
    q, O = torch.empty(2, a.tokens, q_heads, 128, dtype=torch.float16, device="cuda"), torch.empty(2, a.tokens, q_heads, 128, dtype=torch.float16, device="cuda")

    def step():
        for i, (cache, s) in enumerate(layers):
            x = qkv[i]
            tm.tm_paged_append(cache, a.batch, x[:, q_heads:q_heads + heads], x[:, q_heads + heads:], rope=rope, Q=x[:, :q_heads], Q_out=q[i])
            tm.tm_paged_attn(q[i], cache, a.batch, O[i], SCALE)

    a.batch.table.copy_(b.batch.table)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        qkv.normal_()
        a.batch.positions.add_(torch.tensor([1, 70, 3], dtype=torch.int32, device="cuda"))
        held = [t.clone() for _, s in layers for t in (s.k, s.v, s.pairs)]
        O.fill_(float("nan"))
        graph.replay()
        got, stored = O.clone(), [t.clone() for _, s in layers for t in (s.k, s.v, s.pairs)]
        for t, h in zip([t for _, s in layers for t in (s.k, s.v, s.pairs)], held):
            t.view(torch.uint8).copy_(h.view(torch.uint8))
        O.fill_(float("nan"))
        step()
        assert torch.equal(got, O) and not torch.isnan(O).any()
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(stored, [t for _, s in layers for t in (s.k, s.v, s.pairs)]))


def test_serving_steps_against_the_contiguous_cache(tm):
    """A prompt in chunks and decoding steps after it, two sequences: what is stored and what comes out, beside tm_kv_append and tm_attn_prefill / tm_attn_decode."""
    import torch
    heads, q_heads, page = 2, 8, 64
    for bits in (8, 4):
        k, v, pairs = tm.tm_paged_pool(12, heads, page, bits)
        cache = tm.tm_paged_create(k, v, pairs)
        slab = tm.tm_kv_create(2, heads, 384, bits)
        table = _dev(np.random.default_rng(0).permutation(12).reshape(2, 6).astype(np.int32))
        at = torch.zeros(2, dtype=torch.int32, device="cuda")
        for n in (100, 37, 1, 1, 8, 1):
            Q, K, V = (torch.randn(2, n, h, 128, device="cuda").half() for h in (q_heads, heads, heads))
            batch = tm.PagedBatch(table, torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda"), at, max_count=n)
            tm.tm_paged_append(cache, batch, K.view(2 * n, heads, 128), V.view(2 * n, heads, 128))
            tm.tm_kv_append(slab, K, V, at)
            O, P = torch.empty(2 * n, q_heads, 128, dtype=torch.float16, device="cuda"), torch.empty(2, n, q_heads, 128, dtype=torch.float16, device="cuda")
            tm.tm_paged_attn(Q.view(2 * n, q_heads, 128), cache, batch, O, SCALE)
            tm.tm_attn_prefill(Q, slab, at, P, SCALE)
            at += n
            # two results that are each within 2^-11 (|O| + A) of the true one; A is at most the largest |V^| met, below 6 here
            assert (O.float() - P.view_as(O).float()).abs().max() <= 2 * 1.125 * 2.0 ** -11 * 12
        slab.close()


def test_refusals(tm):
    import torch
    s = Setup(tm, 8, 32, 2, [4], [0], q_heads=4)
    O = torch.empty_like(s.Q)
    for call, error, text in [(lambda: tm.tm_paged_attn(s.Q, s.cache, s.batch, O, 0.0), tm.TmError, "scale"),
                              (lambda: tm.tm_paged_attn(s.Q, s.cache, s.batch, O, float("nan")), tm.TmError, "scale"),
                              (lambda: tm.tm_paged_attn(s.Q[:, :3], s.cache, s.batch, O[:, :3].contiguous(), 1.0), tm.TmError, "q_heads"),
                              (lambda: tm.tm_paged_attn(s.Q, s.cache, s.batch, O[:3], 1.0), ValueError, "Q and O"),
                              (lambda: tm.tm_paged_attn(s.Q, s.cache, s.batch, torch.empty(4, 5, 128, dtype=torch.float16, device="cuda")[:, :4], 1.0), ValueError, "contiguous"),
                              (lambda: tm.tm_paged_attn(s.Q.float(), s.cache, s.batch, O, 1.0), TypeError, "float16"),
                              (lambda: tm.tm_get_paged_plan(s.cache, s.batch, -1, 4), ValueError, "tokens"),
                              (lambda: tm.tm_get_paged_plan(s.cache, s.batch, 1 << 30, 8), tm.TmError, "tokens")]:
        with pytest.raises(error, match=text):
            call()
    assert tm.tm_paged_attn(s.Q[:0], s.cache, s.batch, O[:0], 1.0).shape[0] == 0
    s.cache.close()
    with pytest.raises(ValueError, match="freed"):
        tm.tm_paged_attn(s.Q, s.cache, s.batch, O, 1.0)
