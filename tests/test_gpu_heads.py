"""GPU parity of norms of heads with the rotation, and of positions of several axes (tm_heads_apply, tm_rope_create_axes, tm_paged_append_heads), against the 64-bit oracle.

A result is one rounding to fp16 through fp32 (2^-11 of the value, 2^-25 below the normal numbers, 2^-24 of it on the way) of what 64 bits give; sines and cosines are right to 1e-11 of
the pair they turn."""
import sys

import numpy as np
import pytest

from oracle import oracle_paged as op
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


def _near(got, want, size):
    return np.abs(got.astype(np.float64) - want) <= np.maximum(2.0 ** -11 * np.abs(want), 2.0 ** -25) * (1 + 2.0 ** -12) + 1e-10 * size


def _axis(pairs, axes):
    return [(i * 5 + i // 3) % axes for i in range(pairs - 1)] + [axes - 1]


class Heads:
    def __init__(self, tm, tokens, q_heads, k_heads, dim, rot=0, layout="half", axes=1, norm="shared", offset=0.0, centred=False, seed=0, eps=1e-5):
        import torch
        rng = np.random.default_rng(seed + tokens + dim)
        self.tm, self.tokens, self.dim, self.inter = tm, tokens, dim, layout == "interleaved"
        heads = q_heads + k_heads
        x = (rng.standard_normal((tokens, heads, dim)) * np.exp(2 * rng.standard_normal((tokens, heads, 1))) + 0.3).astype(np.float16)
        self.x = {"Q": x[:, :q_heads], "K": x[:, q_heads:]}
        self.both = _dev(x)
        self.X = {"Q": self.both[:, :q_heads], "K": self.both[:, q_heads:]}
        self.w, self.norm = {}, {}
        for side, n in (("Q", q_heads), ("K", k_heads)):
            w = (rng.standard_normal((n, dim) if norm == "own" else dim) * 0.5 + 1).astype(np.float16) if norm in ("own", "shared") else None
            self.w[side] = w
            self.norm[side] = tm.HeadNorm(None if w is None else _dev(w), eps=eps, offset=offset, centred=centred) if norm != "none" and n else None
        self.args = dict(eps=eps, offset=offset, centred=centred)
        self.rope = self.positions = None
        if rot:
            self.axis = _axis(rot // 2, axes)
            self.rope = tm.tm_rope_create(rot, layout=int(self.inter), axis=self.axis if axes > 1 else None, amplitude=1.25)
            assert self.rope.axes == axes
            self.pos = rng.integers(-1000, 1 << 20, (tokens, axes))
            self.pos[:1] = (1 << 31) - 1
            self.pos[1:2] = -(1 << 31)
            self.positions = _dev(self.pos.astype(np.int32) if axes > 1 else self.pos[:, 0].astype(np.int32))

    def apply(self, Q_out, K_out, sides="QK", **kw):
        args = {}
        for s, out in (("Q", Q_out), ("K", K_out)):
            if s in sides:
                args |= {s: self.X[s], s + "_out": out, s.lower() + "_norm": self.norm[s]}
        self.tm.tm_heads_apply(rope=self.rope, positions=self.positions, **args, **kw)

    def want(self, side, rows):
        n = self.x[side][rows].astype(np.float64)
        if self.norm[side] is not None:
            n = st.head_norm(n, self.w[side], **self.args)
        size = np.abs(n).max(-1, keepdims=True)
        if self.rope is None:
            return n, size
        f, amp = self.tm.tm_rope_frequencies(self.rope)
        return st.rope_axes(n, self.pos[rows], f, self.axis, amp, self.inter), size


CASES = [
    # tokens, Q heads, K heads, dim, rot, layout, axes, norm, offset, centred
    (1, 1, 1, 128, 128, "half", 1, "shared", 0.0, False),
    (3, 5, 2, 128, 64, "interleaved", 3, "own", 1.0, True),
    (16, 32, 8, 128, 128, "half", 1, "shared", 1.0, False),
    (7, 28, 4, 128, 96, "half", 2, "own", 0.0, False),
    (5, 3, 3, 80, 80, "half", 2, "none", 0.0, False),
    (9, 2, 1, 72, 16, "interleaved", 1, "shared", 0.0, True),             # an odd multiple of eight: the last lane holds eight dimensions
    (4, 17, 1, 8, 0, "half", 1, "shared", 0.0, True),                     # the smallest head, no rotation
    (6, 9, 5, 16, 16, "half", 8, "ones", 0.5, False),                     # as many axes as pairs
    (5, 7, 3, 24, 16, "interleaved", 1, "own", 0.0, False),
    (4, 6, 2, 64, 32, "half", 3, "shared", 0.0, True),
    (3, 3, 1, 256, 256, "half", 3, "own", 1.0, True),
    (3, 3, 2, 248, 192, "interleaved", 2, "shared", 0.0, False),
    (2100, 28, 4, 128, 128, "half", 3, "shared", 0.0, False),             # a wave takes all heads of a token
    (1111, 64, 1, 96, 64, "interleaved", 1, "own", 1.0, True),
]


@pytest.mark.parametrize("tokens, q_heads, k_heads, dim, rot, layout, axes, norm, offset, centred", CASES)
def test_heads(tm, tokens, q_heads, k_heads, dim, rot, layout, axes, norm, offset, centred):
    import torch
    print(f"heads tokens={tokens} {q_heads}/{k_heads} dim={dim} rot={rot} {layout} axes={axes} {norm}", file=sys.stderr, flush=True)
    s = Heads(tm, tokens, q_heads, k_heads, dim, rot, layout, axes, norm, offset, centred)
    # out of one array into rows that lie apart, next to values that stay
    wide = torch.full((tokens, q_heads + k_heads + 3, dim), 7.0, dtype=torch.float16, device="cuda")
    Q, K = wide[:, 1:1 + q_heads], wide[:, 2 + q_heads:2 + q_heads + k_heads]
    s.apply(Q, K)
    rows = np.r_[0:min(tokens, 5), max(tokens - 2, 0):tokens]
    for side, got in (("Q", Q), ("K", K)):
        want, size = s.want(side, rows)
        assert _near(_host(got)[rows], want, size).all()
    assert (wide[:, 0] == 7).all() and (wide[:, 1 + q_heads] == 7).all() and (wide[:, -1] == 7).all()
    if norm == "none" and rot:                                            # the rotation alone is tm_rope_apply, bit for bit
        Y = torch.empty_like(s.both)
        tm.tm_rope_apply(s.both, s.positions, s.rope, Y)
        assert torch.equal(Y[:, :q_heads], Q) and torch.equal(Y[:, q_heads:], K)
    # one side alone; in place
    for sides in "QK":
        alone = {"Q": torch.empty_like(Q), "K": torch.empty_like(K)}
        s.apply(alone["Q"], alone["K"], sides=sides)
        assert torch.equal(alone[sides], {"Q": Q, "K": K}[sides])
    s.apply(s.X["Q"], s.X["K"])
    assert torch.equal(s.both[:, :q_heads], Q) and torch.equal(s.both[:, q_heads:], K)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("norm, centred", [("none", False), ("shared", False), ("own", True)])
def test_every_dimension(tm, layout, norm, centred):
    """Heads of 8 to 256 dimensions, of which none, sixteen, about half or all that can be are turned, more of them than lanes go into; what lies next to them stays."""
    import torch
    for dim in range(8, 257, 8):
        for rot in sorted({0, 16, dim // 32 * 16, dim // 16 * 16}):
            if rot > dim or (rot == 0 and norm == "none"):
                continue
            q_heads, k_heads = 1 + dim // 8 % 5, 3 + dim // 8 % 7
            s = Heads(tm, 2, q_heads, k_heads, dim, rot, layout, 1, norm, 0.5, centred)
            wide = torch.full((2, q_heads + k_heads + 3, dim), 7.0, dtype=torch.float16, device="cuda")
            Q, K = wide[:, 1:1 + q_heads], wide[:, 2 + q_heads:2 + q_heads + k_heads]
            s.apply(Q, K)
            for side, got in (("Q", Q), ("K", K)):
                want, size = s.want(side, np.arange(2))
                assert _near(_host(got), want, size).all(), (dim, rot, side)
            assert (wide[:, 0] == 7).all() and (wide[:, 1 + q_heads] == 7).all() and (wide[:, -1] == 7).all(), (dim, rot)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("axes, rot, dim", [(2, 128, 128), (3, 96, 128), (4, 32, 64), (8, 256, 256)])
def test_axes_of_tm_rope_apply(tm, axes, rot, dim, layout):
    import torch
    rng = np.random.default_rng(rot)
    x, axis = rng.standard_normal((23, 5, dim)).astype(np.float16), _axis(rot // 2, axes)
    pos = rng.integers(-(1 << 31), 1 << 31, (23, axes))
    rope = tm.tm_rope_create(rot, layout=int(layout == "interleaved"), base=500000.0, axis=axis)
    Y = tm.tm_rope_apply(_dev(x), _dev(pos.astype(np.int32)), rope, torch.empty(23, 5, dim, dtype=torch.float16, device="cuda"))
    f, amp = tm.tm_rope_frequencies(rope)
    want = st.rope_axes(x, pos, f, axis, amp, layout == "interleaved")
    assert _near(_host(Y), want, np.abs(x).max()).all() and np.array_equal(_host(Y)[..., rot:], x[..., rot:])
    # the same position on every axis: one axis
    one = tm.tm_rope_create(rot, layout=int(layout == "interleaved"), base=500000.0)
    same = _dev(pos[:, :1].astype(np.int32)).expand(-1, axes).contiguous()
    a, b = tm.tm_rope_apply(_dev(x), same, rope, torch.empty_like(Y)), tm.tm_rope_apply(_dev(x), same[:, 0].contiguous(), one, torch.empty_like(Y))
    assert torch.equal(a, b)


@pytest.mark.parametrize("rot, layout", [(0, "half"), (64, "half"), (128, "interleaved")])
@pytest.mark.parametrize("centred", [False, True])
@pytest.mark.parametrize("tokens", [3, 3000])
def test_one_side_normed(tm, tokens, rot, layout, centred):
    """The other one is turned as tm_rope_apply turns it, bit for bit, and what is not turned is copied bit for bit.  Where the
    turn's sum is NaN both must be NaN: IEEE 754 leaves the sign of a NaN that arithmetic returns undefined (a x - b y and
    a x + (-b) y may give different ones), so it is compared only in the columns that no arithmetic touches."""
    import torch
    s = Heads(tm, tokens, 12, 4, 128, rot, layout, 1, "shared", 0.0, centred)
    s.both[0, 12:, 64:] = torch.tensor([-0.0, float("nan"), float("inf"), -65504.0] * 16, device="cuda").half()
    for side, other in ("QK", "KQ"):
        keep, s.norm[other] = s.norm[other], None
        out = {"Q": torch.empty(tokens, 12, 128, dtype=torch.float16, device="cuda"), "K": torch.empty(tokens, 4, 128, dtype=torch.float16, device="cuda")}
        s.apply(out["Q"], out["K"])
        plain = s.X[other].contiguous()
        if rot:
            tm.tm_rope_apply(s.X[other], s.positions, s.rope, plain)
        same = out[other].view(torch.int16) == plain.view(torch.int16)
        same[..., :rot] |= out[other][..., :rot].isnan() & plain[..., :rot].isnan()
        assert same.all()
        if side == "Q":
            want, size = s.want(side, np.arange(min(tokens, 3)))
            assert _near(_host(out[side])[:3], want, size).all()
        s.norm[other] = keep


def test_heads_of_zeros_infinities_and_nan(tm):
    """A head of zeros is zeros, one with an infinity or a NaN is NaN as the formula has it, and no head touches another."""
    import torch
    x = torch.randn(2, 4, 128, device="cuda").half()
    x[0, 0], x[0, 1, 5], x[1, 2, 77], x[1, 3] = 0, float("inf"), float("nan"), 65504.0
    for centred in (False, True):
        y = torch.empty_like(x)
        tm.tm_heads_apply(K=x, K_out=y, k_norm=tm.HeadNorm(None, eps=1e-6, centred=centred))
        assert (y[0, 0] == 0).all() and torch.isnan(y[0, 1, 5]) and torch.isnan(y[1, 2]).all()
        assert (y[1, 3] == (0 if centred else 1)).all()
        if not centred:
            assert (y[0, 1, :5] == 0).all()                               # a finite value over an infinite norm
        d = x[1, 1].double()
        d = d - d.mean() if centred else d
        want = d / (d.square().mean() + 1e-6).sqrt()
        assert ((y[1, 1].double() - want).abs() <= 2.0 ** -11 * 1.001 * want.abs() + 2.0 ** -25).all()


def test_small_heads_go_by_eps(tm):
    """Heads of the smallest numbers, whose squares fp32 has not: the norm's eps is all that counts, or with a tiny one they count themselves."""
    import torch
    x = torch.full((1, 2, 128), 2.0 ** -24, dtype=torch.float16, device="cuda")
    y = torch.empty_like(x)
    tm.tm_heads_apply(Q=x, Q_out=y, q_norm=tm.HeadNorm(None, eps=2.0 ** -40))
    want = 2.0 ** -24 / (2.0 ** -48 + 2.0 ** -40) ** 0.5
    assert ((y.double() - want).abs() <= 2.0 ** -11 * 1.001 * want).all()
    tm.tm_heads_apply(Q=x, Q_out=y, q_norm=tm.HeadNorm(None, eps=1e-300))
    assert (y == 1).all()


class Pool:
    def __init__(self, tm, bits, page, heads, counts, past, seed=0, **hints):
        import torch
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rng = np.random.default_rng(seed)
        cols = max(-(-(n + p) // page) for n, p in zip(counts, past))
        pages = len(counts) * cols + 2
        self.k, self.v = (torch.randint(0, 256, (pages, heads, page // 32, 512 * bits), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
        self.pairs = torch.randint(-32768, 32768, (pages, heads, page, 2, 2), generator=g, device="cuda", dtype=torch.int16).view(torch.float16)
        self.cache = tm.tm_paged_create(self.k, self.v, self.pairs)
        table = rng.permutation(pages)[:len(counts) * cols].reshape(-1, cols).astype(np.int32)
        offsets = (1 + np.cumsum([0] + list(counts))).astype(np.int32)    # a row before the first sequence
        self.tokens = int(offsets[-1]) + 2                                # and two behind the last
        self.batch = tm.PagedBatch(_dev(table), _dev(offsets), _dev(np.array(past, np.int32)), **hints)
        self.at = np.concatenate([[0]] + [np.arange(p, p + n) for n, p in zip(counts, past)] + [[0, 0]])

    def contents(self):
        return [t.view(__import__("torch").int16) if t.dtype != __import__("torch").uint8 else t for t in (self.k, self.v, self.pairs)]


APPENDS = [
    # counts, positions, max_count, Q heads, KV heads, page, rot, layout, axes, norm
    ([1], [5], 1, 4, 1, 32, 128, "half", 1, "shared"),
    ([1, 1, 1], [0, 31, 64], 1, 32, 8, 64, 128, "half", 1, "own"),
    ([1, 0, 1], [3, 9, 200], 1, 7, 1, 128, 64, "interleaved", 3, "shared"),
    ([5, 3, 1], [30, 0, 100], 5, 8, 2, 32, 96, "half", 2, "shared"),
    ([8, 8], [1, 60], 8, 5, 5, 64, 0, "half", 1, "own"),                   # norms without a rotation
    ([100, 33, 1], [0, 31, 77], 0, 28, 4, 64, 128, "half", 3, "own"),
    ([40, 200], [13, 0], 0, 6, 3, 32, 32, "interleaved", 2, "none"),       # positions of their own without norms
    ([700], [1], 0, 8, 8, 256, 128, "interleaved", 1, "shared"),
    ([64] * 40, list(range(40)), 0, 32, 8, 64, 128, "half", 3, "shared"),  # several KV heads a CTA
]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("counts, past, max_count, q_heads, heads, page, rot, layout, axes, norm", APPENDS)
def test_append_stores_what_heads_apply_gives(tm, bits, counts, past, max_count, q_heads, heads, page, rot, layout, axes, norm):
    """Codes, pairs and queries are bit for bit those of tm_heads_apply followed by tm_paged_append of its keys, in pools of arbitrary bytes, and nothing else changes.  (The norms of the
    two may differ in the last of 53 bits: one value in 2^40 next to the middle between two fp16 numbers.)"""
    import torch
    print(f"append bits={bits} counts={counts[:4]} past={past[:4]} {q_heads}/{heads} page={page} rot={rot} {layout} axes={axes} {norm}", file=sys.stderr, flush=True)
    a, b = (Pool(tm, bits, page, heads, counts, past, seed=3, max_count=max_count) for _ in range(2))
    s = Heads(tm, a.tokens, q_heads, heads, 128, rot, layout, axes, norm, 1.0, norm == "own")
    V = torch.randn(a.tokens, heads, 128, device="cuda").half()
    own = axes == 1 and rot                                               # turned by the sequences' positions
    if own:
        s.positions = _dev(a.at.astype(np.int32))
    Q, K, out = torch.empty(a.tokens, q_heads, 128, dtype=torch.float16, device="cuda"), torch.empty(a.tokens, heads, 128, dtype=torch.float16, device="cuda"), None
    s.apply(Q, K)
    tm.tm_paged_append(a.cache, a.batch, K, V)
    out = torch.full((a.tokens, q_heads + 1, 128), 7.0, dtype=torch.float16, device="cuda")
    tm.tm_paged_append(b.cache, b.batch, s.X["K"], V, rope=s.rope, Q=s.X["Q"], Q_out=out[:, 1:], q_norm=s.norm["Q"], k_norm=s.norm["K"], positions=None if own else s.positions)
    for x, y in zip(a.contents(), b.contents()):
        assert torch.equal(x, y)
    assert torch.equal(out[1:-2, 1:], Q[1:-2]) and (out[:, 0] == 7).all() and (out[[0, -2, -1]] == 7).all()
    # keys alone
    c = Pool(tm, bits, page, heads, counts, past, seed=3, max_count=max_count)
    tm.tm_paged_append(c.cache, c.batch, s.X["K"], V, rope=s.rope, k_norm=s.norm["K"], positions=None if own else s.positions)
    for x, y in zip(a.contents(), c.contents()):
        assert torch.equal(x, y)


def test_text_positions_stand_on_every_axis(tm):
    """A rope of several axes without positions: the sequence's, on all of them."""
    import torch
    a, b = (Pool(tm, 8, 64, 2, [70, 1], [0, 90], seed=1) for _ in range(2))
    x = torch.randn(a.tokens, 8, 128, device="cuda").half()
    out = [torch.empty_like(x) for _ in range(2)]
    many = tm.tm_rope_create(128, axis=_axis(64, 3))
    tm.tm_paged_append(a.cache, a.batch, x[:, :2], x[:, 2:4], rope=many, Q=x, Q_out=out[0])
    tm.tm_paged_append(b.cache, b.batch, x[:, :2], x[:, 2:4], rope=tm.tm_rope_create(128), Q=x, Q_out=out[1])
    assert torch.equal(out[0][1:-2], out[1][1:-2]) and all(torch.equal(p, q) for p, q in zip(a.contents(), b.contents()))


@pytest.mark.parametrize("counts, max_count", [([1, 1], 1), ([3, 70], 0)])
def test_positions_of_their_own_on_one_axis(tm, counts, max_count):
    """What a key is turned by need not be where it is stored (a context that was cut, say)."""
    import torch
    a, b = (Pool(tm, 8, 32, 2, counts, [50, 7], seed=6, max_count=max_count) for _ in range(2))
    x = torch.randn(a.tokens, 8, 128, device="cuda").half()
    at = torch.randint(0, 1 << 30, (a.tokens,), device="cuda", dtype=torch.int32)
    rope = tm.tm_rope_create(96)
    turned, out = torch.empty_like(x), torch.empty_like(x)
    tm.tm_rope_apply(x, at, rope, turned)
    tm.tm_paged_append(a.cache, a.batch, turned[:, :2], x[:, 2:4])
    tm.tm_paged_append(b.cache, b.batch, x[:, :2], x[:, 2:4], rope=rope, Q=x, Q_out=out, positions=at)
    assert torch.equal(out[1:-2], turned[1:-2]) and all(torch.equal(p, q) for p, q in zip(a.contents(), b.contents()))


def test_rows_further_apart_than_32_bits_count(tm):
    import torch
    far = (1 << 30) + 8
    space = torch.empty(2 * far + 4096, dtype=torch.float16, device="cuda")
    X = space.as_strided((3, 2, 128), (far, 128, 1))
    X.copy_(torch.randn(3, 2, 128, device="cuda"))
    pos = torch.tensor([5, 6, 7], dtype=torch.int32, device="cuda")
    rope, norm = tm.tm_rope_create(128), tm.HeadNorm(torch.randn(128, device="cuda").half())
    want = torch.empty(3, 2, 128, dtype=torch.float16, device="cuda")
    tm.tm_heads_apply(rope=rope, positions=pos, Q=X.contiguous(), Q_out=want, q_norm=norm)
    tm.tm_heads_apply(rope=rope, positions=pos, Q=X, Q_out=X, q_norm=norm)
    assert torch.equal(X, want)


def test_heads_in_a_graph_and_on_another_stream(tm):
    import torch
    s = Heads(tm, 50, 8, 2, 128, 128, "half", 3)
    Q, K = torch.empty(50, 8, 128, dtype=torch.float16, device="cuda"), torch.empty(50, 2, 128, dtype=torch.float16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s.apply(Q, K, stream=side)
    side.synchronize()
    first = Q.clone(), K.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.apply(Q, K)
    for i in range(3):                                                    # follows what the arrays hold at the replay
        s.positions.add_(i)
        Q.fill_(1), K.fill_(1)
        g.replay()
        torch.cuda.synchronize()
        got = Q.clone(), K.clone()
        s.apply(Q, K)
        assert torch.equal(got[0], Q) and torch.equal(got[1], K) and (i or torch.equal(got[0], first[0]) and torch.equal(got[1], first[1]))


def test_refusals_on_the_device(tm):
    import torch
    x, pos = torch.zeros(4, 2, 128, dtype=torch.float16, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    rope, two = tm.tm_rope_create(128), tm.tm_rope_create(128, axis=[0, 1] * 32)
    w = torch.ones(128, dtype=torch.float16, device="cuda")
    odd = torch.ones(136, dtype=torch.float16, device="cuda")[1:129]
    pool = Pool(tm, 8, 32, 2, [1], [0])
    for call, error, text in [
            (lambda: tm.tm_heads_apply(rope=two, positions=pos, Q=x, Q_out=x), ValueError, "2 axes"),
            (lambda: tm.tm_heads_apply(rope=rope, positions=pos[:, None].expand(4, 2).contiguous(), Q=x, Q_out=x), ValueError, "1 axes"),
            (lambda: tm.tm_rope_apply(x, pos, two, x), ValueError, "2 axes"),
            (lambda: tm.tm_heads_apply(Q=x, Q_out=x, q_norm=tm.HeadNorm(odd)), tm.TmError, "aligned"),
            (lambda: tm.tm_heads_apply(Q=x, Q_out=x, q_norm=tm.HeadNorm(w, eps=0.0)), tm.TmError, "eps"),
            (lambda: tm.tm_heads_apply(Q=x, Q_out=x, q_norm=tm.HeadNorm(w, eps=float("nan"))), tm.TmError, "eps"),
            (lambda: tm.tm_heads_apply(Q=x, Q_out=x, q_norm=tm.HeadNorm(w, offset=float("inf"))), tm.TmError, "offset"),
            (lambda: tm.tm_heads_apply(Q=x, Q_out=x, q_norm=tm.HeadNorm(w[:64])), ValueError, "weight"),
            (lambda: tm.tm_heads_apply(Q=x, Q_out=x, q_norm=tm.HeadNorm(w.float())), TypeError, "float16"),
            (lambda: tm.tm_heads_apply(Q=x, Q_out=x, K=x[:3], K_out=x[:3]), ValueError, "need"),
            (lambda: tm.tm_heads_apply(rope=rope, positions=pos, Q=x[..., :64].contiguous(), Q_out=x[..., :64].contiguous()), tm.TmError, "head_dim"),
            (lambda: tm.tm_paged_append(pool.cache, pool.batch, x, x, q_norm=tm.HeadNorm(w)), ValueError, "without Q"),
            (lambda: tm.tm_paged_append(pool.cache, pool.batch, x, x, positions=pos), ValueError, "without a rope"),
            (lambda: tm.tm_paged_append(pool.cache, pool.batch, x, x, rope=two, positions=pos), ValueError, "2 axes"),
            (lambda: tm.tm_paged_append(pool.cache, pool.batch, x, x, k_norm=tm.HeadNorm(w, eps=-1.0)), tm.TmError, "eps")]:
        with pytest.raises(error, match=text):
            call()
    tm.tm_heads_apply(rope=rope, positions=pos[:0], Q=x[:0], Q_out=x[:0], q_norm=tm.HeadNorm(w))      # no tokens: nothing to do
    assert (x == 0).all()
