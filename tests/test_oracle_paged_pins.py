"""Pins of the oracle for rotary positions and paged attention: closed forms, identities and the contiguous oracle."""
import math

import numpy as np
import pytest

from oracle import oracle_attn as oa
from oracle import oracle_paged as op
from workloads import attn as wa


def test_rope_of_a_quarter_turn_swaps_the_pair():
    x = np.array([[[1.0, 2.0, 3.0, 4.0]]])
    f = [math.pi / 2, 0.0]
    assert np.allclose(op.rope(x, [1], f), [[[-3.0, 2.0, 1.0, 4.0]]], atol=1e-15)                       # pairs (0, 2), (1, 3)
    assert np.allclose(op.rope(x, [1], f, interleaved=True), [[[-2.0, 1.0, 3.0, 4.0]]], atol=1e-15)     # pairs (0, 1), (2, 3)
    assert np.allclose(op.rope(x, [2], f), [[[-1.0, 2.0, -3.0, 4.0]]], atol=1e-15)
    assert np.allclose(op.rope(x, [-1], f, amp=2.0), [[[6.0, 4.0, -2.0, 8.0]]], atol=1e-14)


def test_rope_keeps_the_rest_and_depends_on_distance_only():
    rng = np.random.default_rng(0)
    f, _ = op.frequencies(16)
    q, k = rng.standard_normal((2, 1, 1, 24))
    y = op.rope(q, [77], f)
    assert np.array_equal(y[..., 16:], q[..., 16:])
    for inter in (False, True):
        dots = [float((op.rope(q, [p + 9], f, interleaved=inter) * op.rope(k, [p], f, interleaved=inter)).sum()) for p in (0, 5, 1 << 20, (1 << 31) - 10)]
        assert np.allclose(dots, dots[0], atol=1e-9)


def test_angles_are_reduced_without_loss():
    # 2^30 * f for f = 2 pi / 2^20 (as a double): the double is off by d from the true value, so the angle is 2^30 * d
    f = 2 * math.pi / 2 ** 20
    d = float(op.Fraction(f) - op._TWO_PI / 2 ** 20)
    a = op.angles([1 << 30], [f])[0, 0]
    a = a - 2 * math.pi if a > 3 else a
    assert abs(a - d * 2 ** 30) < 1e-15 and abs(a) < 1e-6


def test_frequency_rules():
    plain, one = op.frequencies(64, 10000.0)
    assert one == 1.0 and plain[0] == 1.0 and abs(plain[16] - 0.01) < 1e-12
    assert np.allclose(op.frequencies(64, 10000.0, "linear", 4.0)[0], plain / 4)
    # the last pair of the base rule turns as slowly as under the linear rule
    assert np.isclose(op.frequencies(64, 10000.0, "base", 8.0)[0][-1], plain[-1] / 8) and op.frequencies(64, 10000.0, "base", 8.0)[0][0] == 1.0
    w = op.frequencies(64, 10000.0, "wavelength", 8.0, 8192, 1.0, 4.0)[0]
    turns = 8192 * plain / (2 * math.pi)
    assert np.allclose(w[turns > 4], plain[turns > 4]) and np.allclose(w[turns < 1], plain[turns < 1] / 8)
    between = (turns > 1) & (turns < 4)
    assert between.any() and (w[between] < plain[between]).all() and (w[between] > plain[between] / 8).all()
    r, amp = op.frequencies(64, 10000.0, "ramp", 16.0, 4096, 1.0, 32.0)
    assert np.isclose(amp, 0.1 * math.log(16) + 1) and r[0] == plain[0] and np.isclose(r[-1], plain[-1] / 16) and (np.diff(r) < 0).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_paged_attention_is_the_contiguous_one(bits):
    B, Hq, Hkv, T, page, n = 2, 4, 2, 96, 32, 3
    Q, K, V, _ = wa.draw(B, Hq, Hkv, T, seed=3)
    rng = np.random.default_rng(4)
    Qc = rng.standard_normal((B, n, Hq, 128)).astype(np.float16)
    kq, vq = oa.kv_quantise(K, bits), oa.kv_quantise(V, bits)
    want = oa.attn_prefill(Qc, *kq, *vq, [T - n, 40], [n, n], 0.1)
    # the same tokens in pages 5, 1, 3 and 0, 2, 4 of a pool
    table = np.array([[5, 1, 3], [0, 2, 4]])
    arrays = []
    for a in (*kq, *vq):
        p = np.empty((6, Hkv, page, *a.shape[3:]), a.dtype)
        for b in range(B):
            for i in range(3):
                p[table[b, i]] = a[b, :, i * page:(i + 1) * page]
        arrays.append(p)
    got = op.attention(Qc.reshape(B * n, Hq, 128), arrays, table, [0, n, 2 * n], [T - n, 40], 0.1)[0]
    assert np.abs(got.reshape(want.shape) - want).max() <= 2 ** -11 * np.abs(want).max()
    # a page that does not exist holds no tokens
    table[0, 1] = 99
    holes = op.attention(Qc[0], arrays, table[:1], [0, n], [T - n], 0.1)[0]
    keep = np.r_[0:32, 64:96]
    less = oa.attn_decode(Qc[:1, 2], *[a[:1, :, keep] for a in (*kq, *vq)], [64], 0.1)
    assert np.abs(holes[2] - less[0]).max() <= 2 ** -11 * np.abs(less).max()
