"""GPU parity of rotary positions and the paged cache (tm_paged.h) against the 64-bit oracle: rotation to the nearest fp16 value, codes and read-back bit for
bit, nothing touched besides."""
import sys

import numpy as np
import pytest

from oracle import oracle_attn as oa
from oracle import oracle_paged as op

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tm():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_2508_15601_amd as tm
    tm.load_library()
    return tm


def _say(msg):
    print(msg, file=sys.stderr, flush=True)


def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _host(t):
    import torch
    torch.cuda.synchronize()
    return t.cpu().numpy()


LAYOUTS = {"half": 0, "interleaved": 1}
RULES = {"plain": {}, "linear": dict(factor=4.0), "base": dict(factor=8.0), "wavelength": dict(factor=8.0, original_len=8192, low=1.0, high=4.0),
         "ramp": dict(factor=16.0, original_len=4096, low=1.0, high=32.0)}


def _rope(tm, rot, layout="half", rule="plain", base=10000.0, **kw):
    return tm.tm_rope_create(rot, layout=LAYOUTS[layout], base=base, scaling=list(RULES).index(rule), **RULES[rule], **kw)


def _near(got, want, slack):
    """One rounding to fp16 through fp32 of a value that is itself off by at most `slack`: half a step of fp16 (2^-11 of the value, 2^-25 below the normal
    numbers) and half one of fp32."""
    want = np.asarray(want, np.float64)
    return np.abs(got.astype(np.float64) - want) <= np.maximum(2.0 ** -11 * np.abs(want), 2.0 ** -25) * (1 + 2.0 ** -12) + slack


# ------------------------------------------------------------------------------------------------------------- rope

@pytest.mark.parametrize("rule", list(RULES))
@pytest.mark.parametrize("rot", [16, 96, 128])
def test_frequencies_follow_the_rules(tm, rot, rule):
    rope = _rope(tm, rot, rule=rule, base=500000.0)
    f, amp = tm.tm_rope_frequencies(rope)
    want, wamp = op.frequencies(rot, 500000.0, rule, **RULES[rule])
    assert np.allclose(f, want, rtol=1e-12, atol=0) and abs(amp - wamp) < 1e-12
    rope.close()


FAR = [0, 1, 2, 1000, 131071, 1 << 20, (1 << 31) - 1, -1, -(1 << 31), 77777]


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("tokens, heads, dim, rot", [(1, 1, 16, 16), (10, 3, 24, 16), (10, 5, 128, 128), (10, 7, 128, 32), (7, 40, 128, 96), (9, 2, 256, 256),
                                                     (10, 9, 72, 64), (300, 8, 128, 128), (10, 70, 64, 64), (2100, 64, 128, 64)])
def test_rope(tm, tokens, heads, dim, rot, layout):
    """Every position an int32 can hold, with angles reduced exactly; parts of a head, head dimensions that are odd multiples of eight."""
    import torch
    _say(f"rope tokens={tokens} heads={heads} dim={dim} rot={rot} {layout}")
    rng = np.random.default_rng(tokens + dim)
    x = rng.standard_normal((tokens, heads, dim)).astype(np.float16)
    pos = np.array((FAR * (tokens // len(FAR) + 1))[:tokens], np.int64)
    pos[len(FAR):] = rng.integers(0, 1 << 20, max(tokens - len(FAR), 0))
    rope = _rope(tm, rot, layout, rule="ramp" if heads == 7 else "plain")
    f, amp = tm.tm_rope_frequencies(rope)
    X, P = _dev(x), _dev(pos.astype(np.int32))
    Y = torch.full_like(X, float("nan"))
    assert tm.tm_rope_apply(X, P, rope, Y) is Y
    some = np.r_[0:min(tokens, 12), max(tokens - 3, 0):tokens]              # the oracle reduces angles in rational arithmetic: a sample
    y = _host(Y)
    assert _near(y[some], op.rope(x[some], pos[some], f, amp, layout == "interleaved"), 1e-9).all()
    # and all of it against doubles (angles up to 2^31 are off by 2^31 * 2^-53 there)
    a = torch.from_numpy(pos).double()[:, None] * torch.tensor(f, dtype=torch.float64)
    c, s = (a.cos() * amp).numpy()[:, None], (a.sin() * amp).numpy()[:, None]
    i0 = np.arange(rot // 2) * (2 if layout == "interleaved" else 1)
    i1 = i0 + (1 if layout == "interleaved" else rot // 2)
    want = x.astype(np.float64)
    want[..., i0], want[..., i1] = x[..., i0] * c - x[..., i1] * s, x[..., i1] * c + x[..., i0] * s
    assert _near(y, want, 1e-5).all() and np.array_equal(y[..., rot:], x[..., rot:])
    # in place, and out of and into rows that lie apart
    Z = X.clone()
    tm.tm_rope_apply(Z, P, rope, Z)
    wide = torch.full((tokens, heads + 3, dim), 7.0, dtype=torch.float16, device="cuda")
    wide[:, 1:heads + 1] = X
    out = torch.full((tokens, heads + 2, dim), 7.0, dtype=torch.float16, device="cuda")
    tm.tm_rope_apply(wide[:, 1:heads + 1], P, rope, out[:, 2:])
    assert torch.equal(Z, Y) and torch.equal(out[:, 2:], Y) and (out[:, :2] == 7).all()
    rope.close()


def _near_quarters(pos, around, tries=4000):
    """Frequencies near `around` whose angle at position `pos` is next to a whole number of quarter turns: (f, that number modulo 4, the angle beyond it), the next of the first `tries`."""
    quarter = op._TWO_PI / 4
    out = []
    for f0 in around:
        k0 = round(op.Fraction(pos) * op.Fraction(f0) / quarter)
        best = None
        for k in range(k0, k0 + tries):
            f = float(k * quarter / pos)
            rest = op.Fraction(pos) * op.Fraction(f) - k * quarter
            if best is None or abs(rest) < abs(best[2]):
                best = (f, k % 4, rest)
        out.append(best)
    return out


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("pos", [(1 << 31) - 1, -(1 << 31), (1 << 24) + 1, 131072])
def test_rope_angles_at_the_ends_of_what_is_accepted(tm, pos, layout):
    """Sines and cosines are right to 1e-11 at every int32 position and for every frequency up to the largest accepted one.  Next to a whole number of quarter turns one of
    the two is next to zero, where fp16 resolves it: of a pair (16384, 0) it leaves 16384 times the angle beyond the quarters, which is known as a rational number."""
    import torch
    found = _near_quarters(pos, [1.0, 0.37, 3e-3, 2e-5, 2500.0, 31415.9, -0.73, 999000.0])
    f = [x[0] for x in found]
    _say(f"rope at {pos}: angles beyond the quarters {[float(x[2]) for x in found]}")
    rope = tm.tm_rope_create(16, layout=LAYOUTS[layout], frequencies=f)
    x = np.zeros((1, 1, 16), np.float16)
    first = np.arange(8) * 2 if layout == "interleaved" else np.arange(8)
    second = first + (1 if layout == "interleaved" else 8)
    x[0, 0, first] = 16384.0
    y = _host(tm.tm_rope_apply(_dev(x), _dev(np.array([pos], np.int32)), rope, torch.empty(1, 1, 16, dtype=torch.float16, device="cuda")))[0, 0]
    # of the quarters 0 .. 3: (cos, sin) = (1, r), (-r, 1), (-1, -r), (r, -1) for a small rest r
    small = np.array([(-1 if k in (1, 2) else 1) * 16384 * np.sin(float(r)) for _, k, r in found])
    large = np.array([(-1 if k in (2, 3) else 1) * 16384 * np.cos(float(r)) for _, k, r in found])
    odd = np.array([k % 2 for _, k, _ in found], bool)
    got_small, got_large = np.where(odd, y[first], y[second]), np.where(odd, y[second], y[first])
    assert _near(got_small, small, 16384e-11).all() and _near(got_large, large, 16384e-11).all(), (got_small, small)
    rope.close()


def test_rope_of_more_tokens_than_a_launch_takes(tm):
    """A wave a token: 2^26 tokens are the threads of a launch."""
    import torch
    n = (1 << 26) + 12345
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    X = torch.randn(n, 1, 16, generator=g, device="cuda", dtype=torch.float16)
    P = torch.arange(n, dtype=torch.int32, device="cuda")
    rope = _rope(tm, 16)
    f, amp = tm.tm_rope_frequencies(rope)
    Y = torch.full_like(X, float("nan"))
    tm.tm_rope_apply(X, P, rope, Y)
    some = np.r_[0:3, (1 << 26) - 6:(1 << 26) + 3, n - 3:n]
    assert _near(_host(Y[some]), op.rope(_host(X[some]), some, f, amp), 1e-9).all()
    Z, half = torch.empty_like(X), n // 2
    tm.tm_rope_apply(X[:half], P[:half], rope, Z[:half])
    tm.tm_rope_apply(X[half:], P[half:], rope, Z[half:])
    assert torch.equal(Y, Z)
    rope.close()


def test_rope_own_frequencies_and_special_values(tm):
    import torch
    f = np.array([0.0, 1.0, -0.25, 2 * np.pi, 3.0, 1e-9, 1e5, 0.5])
    rope = tm.tm_rope_create(16, frequencies=f, amplitude=1.25)
    x = np.random.default_rng(0).standard_normal((3, 1, 16)).astype(np.float16)
    x[1, 0, :4] = [np.inf, -np.inf, np.nan, 65504]
    x[2] = np.array([2.0 ** -24, 2.0 ** -20, 2.0 ** -15, 0.0] * 4)
    pos = [3, 0, 100000]
    y = _host(tm.tm_rope_apply(_dev(x), _dev(np.array(pos, np.int32)), rope, torch.empty(3, 1, 16, dtype=torch.float16, device="cuda")))
    with np.errstate(all="ignore"):
        want = op.rope(x, pos, f, 1.25)
    rows = [0, 2]
    assert _near(y[rows], want[rows], 1e-9).all()
    assert np.isinf(y[1, 0, 0]) and np.isnan(y[1, 0, 2]) and np.isnan(y[1, 0, 10]) and np.isinf(y[1, 0, 3])       # 65504 * 1.25 is out of range
    with pytest.raises(tm.TmError, match="head_dim"):
        tm.tm_rope_apply(torch.zeros(1, 1, 12, dtype=torch.float16, device="cuda"), _dev(np.zeros(1, np.int32)), rope, torch.zeros(1, 1, 12, dtype=torch.float16, device="cuda"))
    rope.close()
    with pytest.raises(ValueError, match="freed"):
        tm.tm_rope_apply(_dev(x), _dev(np.array(pos, np.int32)), rope, _dev(x))


# ---------------------------------------------------------------------------------------------------- append and read

class Pool:
    """A pool filled with arbitrary bytes (NaN scales among them) and a batch over it."""

    def __init__(self, tm, bits, page, heads, counts, positions, max_pages, seed=0, before=0, behind=0, tables=None, **hints):
        import torch
        rng = np.random.default_rng(seed)
        B = len(counts)
        self.pages = B * max_pages + 2
        self.k, self.v = (_dev(rng.integers(0, 256, (self.pages, heads, page // 32, 512 * bits), np.uint8)) for _ in range(2))
        self.pairs = _dev(rng.integers(0, 1 << 16, (self.pages, heads, page, 2, 2), np.uint16).view(np.float16))
        self.table = rng.permutation(self.pages)[:B * max_pages].reshape(B, max_pages).astype(np.int32) if tables is None else tables
        self.offsets = (before + np.cumsum([0] + list(counts))).astype(np.int32)
        self.counts, self.positions, self.tokens = counts, positions, int(self.offsets[-1]) + behind
        self.page, self.bits, self.heads, self.cap = page, bits, heads, max_pages * page
        self.cache = tm.tm_paged_create(self.k, self.v, self.pairs)
        self.batch = tm.PagedBatch(_dev(self.table), _dev(self.offsets), _dev(np.asarray(positions, np.int32)), **hints)

    def arrays(self):
        return [a.copy() for a in op.unpack_pool(_host(self.k), _host(self.v), _host(self.pairs))]

    def slots(self):
        """(row, page, slot, position) of every new token that has a place."""
        for b, n in enumerate(self.counts):
            for i in range(n):
                p = int(self.positions[b]) + i
                if 0 <= p < self.cap and 0 <= self.table[b, p // self.page] < self.pages:
                    yield int(self.offsets[b]) + i, self.table[b, p // self.page], p % self.page, p

    def row_positions(self):
        return np.concatenate([np.arange(n) + int(p) for n, p in zip(self.counts, self.positions)]) if sum(self.counts) else np.zeros(0, int)


def _bits(a):
    return a.view(np.uint16) if a.dtype == np.float16 else a


def _same(name, got, want):
    off = np.argwhere(_bits(got) != _bits(want))
    assert not len(off), f"{name}: {len(off)} differ, first at {off[0].tolist()}: {got[tuple(off[0])]} for {want[tuple(off[0])]}"


def _check_append(tm, pool, rope=None, q_heads=3, seed=1):
    import torch
    rng = np.random.default_rng(seed)
    qkv = _dev(rng.standard_normal((pool.tokens, q_heads + 2 * pool.heads, 128)).astype(np.float16))
    Q, K, V = qkv.split((q_heads, pool.heads, pool.heads), 1)
    k = _host(K).copy()
    want = pool.arrays()
    out = torch.full((pool.tokens, q_heads + 1, 128), 9.0, dtype=torch.float16, device="cuda")
    if rope is not None:
        first, last = int(pool.offsets[0]), int(pool.offsets[-1])
        pos = np.zeros(pool.tokens, np.int32)
        pos[first:last] = pool.row_positions()
        turned = torch.empty_like(qkv)
        tm.tm_rope_apply(qkv, _dev(pos), rope, turned)                     # checked above
        k = _host(turned[:, q_heads:q_heads + pool.heads])
        assert tm.tm_paged_append(pool.cache, pool.batch, K, V, rope=rope, Q=Q, Q_out=out[:, 1:]) is not None
        o = _host(out)
        _same("queries", np.ascontiguousarray(o[first:last, 1:]), np.ascontiguousarray(_host(turned[first:last, :q_heads])))
        assert (o[:, :1] == 9).all() and (o[:first] == 9).all() and (o[last:] == 9).all()
    else:
        tm.tm_paged_append(pool.cache, pool.batch, K, V)
    v = _host(V)
    for row, page, slot, _ in pool.slots():
        for h in range(pool.heads):
            for base, x in ((0, k), (3, v)):
                q, s, z = oa.kv_quantise(x[row, h], pool.bits)
                want[base][page, h, slot], want[base + 1][page, h, slot], want[base + 2][page, h, slot] = q, s, z
    for name, got, w in zip(("key codes", "key scales", "key zeros", "value codes", "value scales", "value zeros"), pool.arrays(), want):
        _same(name, got, w)                                                # the new tokens' codes and pairs, and every other byte as it was


def _check_read(tm, pool):
    import torch
    K, V = (torch.full((pool.tokens, pool.heads, 128), 9.0, dtype=torch.float16, device="cuda") for _ in range(2))
    tm.tm_paged_read(pool.cache, pool.batch, K, V)
    want = [np.full((pool.tokens, pool.heads, 128), 9.0, np.float16) for _ in range(2)]
    pos = pool.row_positions()
    for w in want:
        rows = np.arange(len(pos)) + int(pool.offsets[0])
        w[rows[(pos >= 0) & (pos < pool.cap)]] = 0.0                       # on a page that is none of the pool's
    a = pool.arrays()
    with np.errstate(all="ignore"):
        for row, page, slot, _ in pool.slots():
            for w, i in zip(want, (0, 3)):
                w[row] = ((a[i][page, :, slot].astype(np.float32) - a[i + 2][page, :, slot].astype(np.float32)[:, None]) * a[i + 1][page, :, slot].astype(np.float32)[:, None]).astype(np.float16)
    for got, w in zip((_host(K), _host(V)), want):
        nan = np.isnan(w)
        assert np.array_equal(np.isnan(got), nan) and np.array_equal(got[~nan], w[~nan])


SHAPES = [
    # page, heads, counts, positions, table columns
    (32, 1, [1], [0], 1),
    (32, 2, [1, 1, 1], [31, 32, 95], 3),                                   # decoding: last slot of a page, first of the next, last of all
    (64, 3, [5, 0, 33, 64], [0, 7, 40, 64], 2),                            # runs that begin and end inside one, a sequence without new tokens
    (128, 1, [128, 100, 1], [0, 27, 255], 2),
    (256, 2, [200, 3], [30, 509], 2),                                      # the last three slots there are
    (1024, 1, [40], [1000], 2),
    (32, 1, [70, 10, 5], [-3, 90, 200], 3),                                # tokens before the first and behind the last slot are dropped
]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("page, heads, counts, positions, cols", SHAPES)
@pytest.mark.parametrize("turn", [None, ("half", 128), ("half", 48), ("interleaved", 64)])
def test_append_and_read(tm, bits, page, heads, counts, positions, cols, turn):
    _say(f"append bits={bits} page={page} heads={heads} counts={counts} positions={positions} rope={turn}")
    pool = Pool(tm, bits, page, heads, counts, positions, cols, seed=sum(counts), before=2, behind=3)
    rope = _rope(tm, turn[1], turn[0], base=500.0) if turn else None
    _check_append(tm, pool, rope)
    _check_read(tm, pool)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("heads, counts, positions, cols", [(9, [1700, 1400, 77], [0, 45, 1000], 14), (8, [900, 803], [5, 64], 8), (3, [1000], [31], 9)])
def test_append_of_prompts(tm, bits, heads, counts, positions, cols):
    """Several KV heads a CTA, with and without queries beside them; heads that do not divide evenly."""
    _say(f"append bits={bits} heads={heads} counts={counts}")
    pool = Pool(tm, bits, 128, heads, counts, positions, cols, seed=heads, before=1, behind=1)
    for rope in (_rope(tm, 96), None):
        _check_append(tm, pool, rope, q_heads=heads)
    _check_read(tm, pool)


@pytest.mark.parametrize("bits", [8, 4])
def test_append_of_a_prompt_without_queries(tm, bits):
    pool = Pool(tm, bits, 64, 5, [7000], [3], 110, seed=bits)
    K, V = (_dev(np.random.default_rng(i).standard_normal((7000, 5, 128)).astype(np.float16)) for i in range(2))
    rope = _rope(tm, 128)
    tm.tm_paged_append(pool.cache, pool.batch, K, V, rope=rope)
    got = pool.arrays()
    tm.tm_paged_append(pool.cache, pool.batch, K, V, rope=rope, Q=K, Q_out=K.clone())
    for a, b in zip(got, pool.arrays()):
        assert np.array_equal(_bits(a), _bits(b))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("batch", [63, 64, 65, 130, 700])
def test_many_sequences(tm, bits, batch):
    """More sequences than a wave has lanes; counts of none, one and a few."""
    _say(f"append batch={batch} bits={bits}")
    rng = np.random.default_rng(batch)
    counts = rng.choice([0, 1, 1, 1, 3], batch).tolist()
    pool = Pool(tm, bits, 32, 1, counts, rng.integers(0, 60, batch).tolist(), 2, seed=batch, before=1, behind=1)
    _check_append(tm, pool, _rope(tm, 64))
    _check_read(tm, pool)


ONE_EACH = SHAPES + [
    (64, 8, [1] * 70, list(range(60, 130)), 3),                            # more sequences than lanes, four waves of vectors a token
    (32, 5, [1, 0, 1], [0, 10, 63], 2),                                    # vectors that do not fill the last wave
    (64, 2, [8, 5, 8, 7, 0, 8], [0, 3, 28, 57, 5, 120], 2),                # drafts: tokens that share bytes of 4-bit values
]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("page, heads, counts, positions, cols", ONE_EACH)
@pytest.mark.parametrize("most, turn, q_heads", [(1, None, 1), (1, ("half", 128), 3), (1, ("half", 48), 40), (1, ("interleaved", 64), 6), (3, ("half", 128), 5), (8, None, 1),
                                                 (9, ("half", 32), 2)])
def test_append_with_a_hint(tm, bits, page, heads, counts, positions, cols, most, turn, q_heads):
    """The hint of one token a sequence or a few, where it is true and where it is not."""
    _say(f"append bits={bits} page={page} heads={heads} counts={counts[:8]} positions={positions[:8]} rope={turn} hint={most}")
    pool = Pool(tm, bits, page, heads, counts, positions, cols, seed=sum(counts), before=2, behind=3, max_count=most)
    rope = _rope(tm, turn[1], turn[0], base=500.0) if turn else None
    _check_append(tm, pool, rope, q_heads=q_heads)
    _check_read(tm, pool)


@pytest.mark.parametrize("bits", [8, 4])
def test_pages_that_do_not_exist(tm, bits):
    _say(f"append bad pages bits={bits}")
    pool = Pool(tm, bits, 32, 2, [96, 40, 1], [0, 20, 64], 3, behind=2)
    table = pool.table.copy()
    table[0, 1], table[1, 0], table[2, 2] = -1, pool.pages, np.int32(-2 ** 31)
    pool.table = table
    pool.batch.table.copy_(_dev(table))
    _check_append(tm, pool, _rope(tm, 128))
    _check_read(tm, pool)
    pool.batch = tm.PagedBatch(pool.batch.table, pool.batch.offsets, pool.batch.positions, max_count=1)
    _check_append(tm, pool, _rope(tm, 128))


def test_extreme_values_are_stored_as_by_the_contiguous_cache(tm):
    import torch
    rng = np.random.default_rng(5)
    x = rng.integers(0, 1 << 16, (2, 70, 2, 128), np.uint16).view(np.float16)
    x = np.where(np.isfinite(x), x, np.float16(0))
    x[:, 1] = (x[:, 1].view(np.uint16) & 0x83ff).view(np.float16)          # subnormal
    x[:, 2] = np.float16(0.37)
    x[:, 3, :, 5], x[:, 4, :, 9] = np.inf, -np.inf
    for bits in (8, 4):
        pool = Pool(tm, bits, 64, 2, [70], [0], 2)
        slab = tm.tm_kv_create(1, 2, 128, bits)
        K, V = _dev(x[0]), _dev(x[1])
        tm.tm_paged_append(pool.cache, pool.batch, K, V)
        tm.tm_kv_append(slab, K[None].contiguous(), V[None].contiguous(), torch.zeros(1, dtype=torch.int32, device="cuda"))
        want = oa.kv_cache_unpack(*tm.tm_kv_download(slab), 1, 2, slab.capacity, bits)
        got = pool.arrays()
        for g, w in zip(got, want):
            joined = np.concatenate([g[p] for p in pool.table[0]], axis=1)
            _same("contiguous cache", np.ascontiguousarray(joined[:, :70]), np.ascontiguousarray(w[0, :, :70]))
        slab.close()


def test_offsets_past_32_bits(tm):
    """A pool whose codes reach beyond 2^32 bytes: pages at its end."""
    import torch
    page, heads, pages = 256, 8, 17000                                     # 256 KiB of key codes a page, 4.4 GB in all
    k, v, pairs = tm.tm_paged_pool(pages, heads, page, 8)
    cache = tm.tm_paged_create(k, v, pairs)
    batch = tm.PagedBatch(_dev(np.array([[pages - 1, pages - 2]], np.int32)), _dev(np.array([0, 300], np.int32)), _dev(np.array([100], np.int32)))
    x = _dev(np.random.default_rng(0).standard_normal((300, 2 * heads, 128)).astype(np.float16))
    tm.tm_paged_append(cache, batch, x[:, :heads], x[:, heads:])
    K, V = (torch.empty(300, heads, 128, dtype=torch.float16, device="cuda") for _ in range(2))
    tm.tm_paged_read(cache, batch, K, V)
    for got, want in ((K, x[:, :heads]), (V, x[:, heads:])):
        w = _host(want).astype(np.float32)
        step = (w.max(-1) - w.min(-1))[..., None] / 255
        # half a step from the code, up to another half where the zero-point was rounded the other way, and the fp16 roundings of scale and result
        assert (np.abs(_host(got).astype(np.float32) - w) <= step * 1.01 + 2.0 ** -9 * np.abs(w)).all()
    # nothing before the two pages was touched
    assert not k[:pages - 2].any() and not pairs[:pages - 2].any()


def test_on_another_stream_and_in_a_graph(tm):
    """Captured once, replayed for other tokens, positions and tables; every replay against an eager call."""
    import torch
    bits, page, heads, q_heads = 4, 32, 2, 4
    pool = Pool(tm, bits, page, heads, [3, 1, 20], [0, 40, 10], 2, max_count=20)
    rope = _rope(tm, 128)
    rng = np.random.default_rng(0)
    Q, K, V = (_dev(rng.standard_normal((24, n, 128)).astype(np.float16)) for n in (q_heads, heads, heads))
    Qo, Kb, Vb = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)

    def step():
        tm.tm_paged_append(pool.cache, pool.batch, K, V, rope=rope, Q=Q, Q_out=Qo)
        tm.tm_paged_read(pool.cache, pool.batch, Kb, Vb)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for shift in (0, 1, 7):
        K.copy_(torch.roll(K, 1, 0))
        Q.mul_(0.5)
        pool.batch.positions.add_(shift)
        pool.batch.table.copy_(torch.roll(pool.batch.table, 1, 0))
        for t in (Qo, Kb, Vb):
            t.fill_(float("nan"))
        graph.replay()
        got = [t.clone() for t in (Qo, Kb, Vb)]
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (Qo, Kb, Vb)))
        assert not any(torch.isnan(t).any() for t in got)


def test_refusals_on_the_device(tm):
    import torch
    pool = Pool(tm, 8, 32, 2, [4], [0], 1)
    x = torch.zeros(4, 2, 128, dtype=torch.float16, device="cuda")
    rope, wide = _rope(tm, 64), _rope(tm, 256)
    for call, error, text in [
            (lambda: tm.tm_paged_append(pool.cache, pool.batch, x, x, Q=x, Q_out=x), tm.TmError, "rope"),
            (lambda: tm.tm_paged_append(pool.cache, pool.batch, x, x, rope=rope, Q=x), ValueError, "together"),
            (lambda: tm.tm_paged_append(pool.cache, pool.batch, x, x, rope=wide), tm.TmError, "128 dimensions"),
            (lambda: tm.tm_paged_append(pool.cache, pool.batch, x.float(), x), TypeError, "float16"),
            (lambda: tm.tm_paged_append(pool.cache, pool.batch, x.transpose(0, 1).contiguous().transpose(0, 1), x), ValueError, "contiguous heads"),
            (lambda: tm.tm_paged_append(pool.cache, pool.batch, x[:1].expand(4, 2, 128), x), ValueError, "overlap"),
            (lambda: tm.tm_paged_read(pool.cache, pool.batch, x[:, :, :64], x), ValueError, "K must be"),
            (lambda: tm.tm_paged_create(pool.k, pool.v, pool.pairs, torch.zeros(1000, dtype=torch.uint8, device="cuda")), tm.TmError, "workspace"),
            (lambda: tm.tm_rope_apply(x, torch.zeros(4, dtype=torch.int64, device="cuda"), rope, x), TypeError, "int32"),
            (lambda: tm.tm_rope_apply(x, torch.zeros(4, dtype=torch.int32, device="cuda"), wide, x), tm.TmError, "head_dim")]:
        with pytest.raises(error, match=text):
            call()
    odd = torch.zeros(4 * 2 * 128 + 8, dtype=torch.float16, device="cuda")[4:4 + 1024].view(4, 2, 128)
    with pytest.raises(tm.TmError, match="16-byte"):
        tm.tm_paged_append(pool.cache, pool.batch, odd, x)
    tm.tm_paged_append(pool.cache, pool.batch, x[:0], x[:0])               # no tokens: nothing to do
    pool.cache.close()
    with pytest.raises(ValueError, match="freed"):
        tm.tm_paged_append(pool.cache, pool.batch, x, x)
