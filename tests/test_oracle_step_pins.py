"""Pins of the oracle for norms of heads, positions of several axes, pages from lengths and attention in a window: closed forms, identities, small cases by hand."""
import math

import numpy as np

from oracle import oracle_attn as oa
from oracle import oracle_paged as op
from oracle import oracle_step as st


def test_norms_in_closed_form():
    x = np.array([[[3.0, -4.0, 0.0, 0.0]]])
    assert np.allclose(st.head_norm(x, eps=0.75), [[[3 / math.sqrt(7), -4 / math.sqrt(7), 0, 0]]])                  # 25 / 4 + 0.75 = 7
    w = np.array([1.0, 2.0, 3.0, 4.0])
    assert np.allclose(st.head_norm(x, w, eps=0.75, offset=1.0), [[[6 / math.sqrt(7), -12 / math.sqrt(7), 0, 0]]])
    y = st.head_norm(np.array([[[1.0, 2.0, 3.0, 4.0], [5.0, 5.0, 5.0, 5.0]]]), np.array([w, w[::-1]]), eps=1e-30, centred=True)
    assert np.allclose(y[0, 0], np.array([-1.5, -0.5, 0.5, 1.5]) / math.sqrt(1.25) * w) and np.array_equal(y[0, 1], np.zeros(4))
    rng = np.random.default_rng(0)
    x = rng.standard_normal((2, 3, 64))
    assert np.allclose(st.head_norm(x * 1000), st.head_norm(x), rtol=1e-5)
    c = st.head_norm(x + 7, centred=True)
    assert np.allclose(c, st.head_norm(x, centred=True)) and np.allclose(c.mean(-1), 0) and np.allclose(c.var(-1), 1, atol=1e-5)


def test_axes():
    rng = np.random.default_rng(1)
    x, f = rng.standard_normal((5, 2, 20)), [0.3, 1.0, 0.01, 2.0]
    pos = rng.integers(0, 1000, (5, 3))
    for inter in (False, True):
        assert np.array_equal(st.rope_axes(x, pos, f, [1] * 4, 1.5, inter), op.rope(x, pos[:, 1], f, 1.5, inter))
        same = np.repeat(pos[:, :1], 3, 1)
        assert np.array_equal(st.rope_axes(x, same, f, [0, 1, 2, 1], interleaved=inter), op.rope(x, pos[:, 0], f, interleaved=inter))
    y = st.rope_axes(np.array([[[1.0, 1.0, 0.0, 0.0]]]), [[1, 2]], [math.pi / 2] * 2, [0, 1])
    assert np.allclose(y, [[[0, -1, 1, 0]]], atol=1e-15)


def test_pages_by_hand():
    table = np.full((3, 4), -1)
    table[0, :2] = 7, 8
    got = st.assign([1, 2, 3, 4, 5], 4, [40, 0, 64], [30, 33, 0], table, 32, 10, 100)
    assert got["table"].tolist() == [[7, 8, 4, -1], [3, 2, -1, -1], [-1] * 4] and got["left"] == 1
    assert got["offsets"] == [0, 30, 63, 63] and got["positions"] == [40, 0, 64] and got["lens"] == [70, 33, 64] and got["lacking"] == [0, 0, 0]
    assert got["slots"][0] == 8 * 32 + 8 and got["slots"][24] == 4 * 32 and got["slots"][30] == 3 * 32 and got["slots"][62] == 2 * 32
    short = st.assign([1, 2], 2, [40, 0, 33], [30, 33, 1], table, 32, 10, 100)                                      # one page, two pages: too many
    assert short["lacking"] == [0, 1, 0] and short["lens"] == [70, 0, 34] and short["left"] == 1 and short["table"][1].tolist() == [-1] * 4
    assert short["slots"][30] == -1 and short["offsets"] == [0, 30, 63, 64]
    pages, n, back = st.release([1, 2, 3, 4, 5], 1, got["table"], 32, 10, first=[33, 0, 0], last=[200, 64, 0])
    assert (pages[:n], back.tolist()) == ([1, 2, 3, 4], [[7, 8, -1, -1], [-1] * 4, [-1] * 4])
    pages, n, back = st.release([1, 2, 3, 4, 5], 1, got["table"], 32, 10)
    assert pages[:n] == [1, 2, 3, 4, 8] and (back == -1).all()                                                      # no room for page 7


def test_window():
    assert st.seen(5, 2, 0) == [4, 5] and st.seen(5, 1, 2) == [0, 1, 5] and st.seen(1, 100, 0) == [0, 1] and st.seen(0, 1, 9) == [0]
    rng = np.random.default_rng(2)
    K, V, Q = rng.standard_normal((3, 64, 2, 128)).astype(np.float16)
    arrays = [a.reshape(2, 32, 2, -1).swapaxes(1, 2) if a.ndim == 3 else a.reshape(2, 32, 2).swapaxes(1, 2)
              for a in (*oa.kv_quantise(K), *oa.kv_quantise(V))]
    table, offsets = np.array([[0, 1]]), [0, 64]
    full = op.attention(Q, arrays, table, offsets, [0], 0.09)
    for window, sinks in ((64, 0), (1, 64), (1000, 7)):
        for a, b in zip(full, st.attention(Q, arrays, table, offsets, [0], 0.09, window, sinks)):
            assert np.allclose(a, b, rtol=1e-12)
    own = st.attention(Q, arrays, table, offsets, [0], 0.09, 1, 0)[0]                                               # a token's own value
    Kd, Vd, _ = op.gather(arrays, table[0], 64)
    assert np.allclose(own, Vd, rtol=1e-12)
