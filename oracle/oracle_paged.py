"""Reference (oracle) for rotary positions and for attention over a paged quantised cache.  TEST INFRASTRUCTURE ONLY: imported by tests/, never by
the GPU library or its binding.

Plain numpy, fp64 throughout, one loop per (sequence, row, head); the quantiser and the order of codes inside a run are those of oracle_attn.

Parity status: rope and the frequency rules are pinned in tests/test_oracle_paged_pins.py (closed forms, complex multiplication, mpmath-free far
positions by exact integer reduction); attention over pages is pinned against oracle_attn on the same tokens laid out contiguously.
"""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

from oracle import oracle_attn as oa


def frequencies(rot: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, original_len: float = 0.0, low: float = 0.0, high: float = 0.0):
    """(f [rot / 2] radians per position, amplitude) by the definitions of include/tm_paged.h, one pair at a time."""
    f, amp = [], 1.0
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2))
    for i in range(rot // 2):
        g = base ** (-2.0 * i / rot)
        if scaling in ("plain", "base"):
            w = None
        elif scaling == "linear":
            w = 0.0
        elif scaling == "wavelength":
            w = (original_len * g / (2 * math.pi) - low) / (high - low)
        else:
            def at(t):
                return rot * math.log(original_len / (2 * math.pi * t)) / (2 * math.log(base))
            a, b = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot - 1)
            w = 1.0 - (i - a) / max(b - a, 0.001)
            amp = 0.1 * math.log(factor) + 1.0
        if w is not None:
            w = min(max(w, 0.0), 1.0)
            g = w * g + (1 - w) * g / factor
        f.append(g)
    return np.array(f), amp


_TWO_PI = Fraction(6283185307179586476925286766559005768394338798750, 10 ** 48)          # 2 pi to 49 decimals


def angles(positions, f) -> np.ndarray:
    """p * f reduced to [0, 2 pi) without loss (exact rational arithmetic): [tokens][pairs]."""
    out = np.empty((len(positions), len(f)))
    for i, p in enumerate(positions):
        for j, x in enumerate(f):
            a = Fraction(int(p)) * Fraction(float(x))
            out[i, j] = float(a - _TWO_PI * (a / _TWO_PI).__floor__())
    return out


def rope(x: np.ndarray, positions, f, amp: float = 1.0, interleaved: bool = False) -> np.ndarray:
    """x [tokens][heads][dim] -> rotated, fp64, not rounded."""
    y = np.asarray(x, np.float64).copy()
    n = len(f)
    a = angles(positions, f)[:, None, :]
    c, s = amp * np.cos(a), amp * np.sin(a)
    i0 = np.arange(n) * 2 if interleaved else np.arange(n)
    i1 = i0 + 1 if interleaved else i0 + n
    x0, x1 = y[..., i0].copy(), y[..., i1].copy()
    y[..., i0] = x0 * c - x1 * s
    y[..., i1] = x1 * c + x0 * s
    return y


def unpack_pool(k, v, pairs):
    """Pool buffers (uint8 [pages][heads][runs][512 * bits], fp16 [pages][heads][page][2][2]) -> the six arrays of oracle_attn.kv_cache_unpack,
    [pages][heads][page](, 128)."""
    pages, heads, runs, size = k.shape
    words = np.ascontiguousarray(pairs).view(np.uint16).astype(np.uint32)
    words = words[..., 0] | (words[..., 1] << 16)
    return oa.kv_cache_unpack(k, v, words, pages, heads, runs * 32, size // 512)


def gather(arrays, table_row, n):
    """Tokens 0 .. n - 1 of a sequence from unpacked pool arrays: keys and values fp64 [n][heads][128], and which of them lie on a page of the pool."""
    Kq, Ks, Kz, Vq, Vs, Vz = arrays
    pages, page = Kq.shape[0], Kq.shape[2]
    t = np.arange(n)
    ids = np.asarray(table_row)[t // page] if n else np.zeros(0, int)
    ok = (ids >= 0) & (ids < pages)
    ids = np.where(ok, ids, 0)
    K = oa.kv_dequant(Kq[ids, :, t % page], Ks[ids, :, t % page], Kz[ids, :, t % page])
    V = oa.kv_dequant(Vq[ids, :, t % page], Vs[ids, :, t % page], Vz[ids, :, t % page])
    return K, V, ok


def attention(Q, arrays, table, offsets, positions, scale: float):
    """(O, A) fp64 [tokens][q_heads][128], NaN in rows that are not to be written.  Row offsets[b] + i at position positions[b] + i attends over the tokens
    0 .. positions[b] + i that lie on a page of the pool; a row with none of them is 0.  A is the same sum over |V^|: what rounding errors of the probabilities are
    measured against."""
    Q = np.asarray(Q, np.float64)
    tokens, Hq, D = Q.shape
    heads, page = arrays[0].shape[1], arrays[0].shape[2]
    cap = table.shape[1] * page
    O, A = np.full(Q.shape, np.nan), np.full(Q.shape, np.nan)
    for b in range(len(positions)):
        n = int(offsets[b + 1]) - int(offsets[b])
        last = min(int(positions[b]) + n, cap)
        if n <= 0 or last <= 0:
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            K, V, ok = gather(arrays, table[b], last)
        for i in range(n):
            p, row = int(positions[b]) + i, int(offsets[b]) + i
            if not 0 <= p < cap:
                continue
            use = np.nonzero(ok[:p + 1])[0]
            for h in range(Hq):
                hk = h // (Hq // heads)
                if not len(use):
                    O[row, h] = A[row, h] = 0.0
                    continue
                x = (K[use, hk] @ Q[row, h]) * float(scale)
                e = np.exp(x - x.max())
                e /= e.sum()
                O[row, h], A[row, h] = e @ V[use, hk], e @ np.abs(V[use, hk])
    return O, A
