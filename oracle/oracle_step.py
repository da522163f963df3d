"""Reference (oracle) for what a server's step does around the paged cache: norms of heads, positions of several axes, pages from lengths, attention in a sliding
window.  TEST INFRASTRUCTURE ONLY: imported by tests/, never by the GPU library or its binding.

Plain numpy in 64 bits and plain Python, one row after another; pinned in tests/test_oracle_step_pins.py.
"""
from __future__ import annotations

import math

import numpy as np

from oracle import oracle_paged as op


def head_norm(x, weight=None, eps=1e-6, offset=0.0, centred=False):
    """x [tokens][heads][dim]; weight [dim] or [heads][dim] or None: fp64, not rounded."""
    x = np.asarray(x, np.float64)
    out = np.empty_like(x)
    for t in range(x.shape[0]):
        for h in range(x.shape[1]):
            v = x[t, h]
            d = v - (math.fsum(v) / len(v) if centred else 0.0)
            w = np.ones(len(v)) if weight is None else np.asarray(weight, np.float64).reshape(-1, len(v))[h if np.ndim(weight) == 2 else 0]
            out[t, h] = d * (offset + w) / math.sqrt(math.fsum(d * d) / len(v) + eps)
    return out


def rope_axes(x, positions, f, axis, amp=1.0, interleaved=False):
    """positions [tokens][axes]; pair i is turned by positions[:, axis[i]].  The pairs of an axis are turned at a time."""
    y = np.asarray(x, np.float64).copy()
    n = len(f)
    for a in sorted(set(axis)):
        turned = op.rope(x, np.asarray(positions)[:, a], f, amp, interleaved)
        for i in range(n):
            if axis[i] == a:
                for d in ((2 * i, 2 * i + 1) if interleaved else (i, i + n)):
                    y[..., d] = turned[..., d]
    return y


def assign(pages, count, lens, counts, table, page, pool_pages, tokens):
    """pages: a list of which the first `count` are free; table [batch][max_pages].  -> dict of what the call writes (slots: row -> slot, others untouched)."""
    table = np.array(table)
    cap = table.shape[1] * page
    free = list(pages[:min(max(count, 0), len(pages))])
    available, asked, at = len(free), 0, 0
    offsets, positions, lens_out, lacking, slots = [0], [], [], [], {}
    for b, (n, new) in enumerate(zip(lens, counts)):
        n, new = min(max(int(n), 0), cap), max(int(new), 0)
        new = min(new, tokens - at)
        have, stop = -(-n // page), min(n + new, cap)
        need = max(-(-stop // page) - have, 0)
        asked += need
        denied = need > 0 and asked > available
        for j in range(have, have + need):
            table[b, j] = -1 if denied else free.pop()
        for i in range(new):
            t = n + i
            entry = table[b, t // page] if t < cap and not denied else -1
            slots[at + i] = int(entry) * page + t % page if 0 <= entry < pool_pages else -1
        at += new
        offsets.append(at)
        positions.append(n)
        lens_out.append(n if denied else stop)
        lacking.append(int(denied))
    return dict(table=table, offsets=offsets, positions=positions, lens=lens_out, lacking=lacking, slots=slots, left=len(free))


def release(pages, count, table, page, pool_pages, first=None, last=None):
    """-> (pages of the list, table): what lies behind the list's end stays."""
    table, pages = np.array(table), list(pages)
    cap, given = table.shape[1] * page, []
    for b in range(table.shape[0]):
        lo = max(int(first[b]), 0) if first is not None else 0
        hi = max(int(last[b]), 0) if last is not None else cap
        for j in range(table.shape[1]):
            if j * page >= lo and (hi >= cap or (j + 1) * page <= hi) and 0 <= table[b, j] < pool_pages:
                given.append(int(table[b, j]))
                table[b, j] = -1
    at = min(max(count, 0), len(pages))
    for id in reversed(given):
        if at < len(pages):
            pages[at] = id
            at += 1
    return pages, at, table


def seen(p, window, sinks):
    """Tokens that the query at position p sees."""
    return [t for t in range(p + 1) if t > p - window or t < sinks]


def attention(Q, arrays, table, offsets, positions, scale, window, sinks):
    """oracle_paged.attention where a row at position p attends over the tokens of seen(p, window, sinks).  (O, A, S): S is the same average over the values' scales, what fp32 sums of
    codes are off by is measured in."""
    Q = np.asarray(Q, np.float64)
    heads, page = arrays[0].shape[1], arrays[0].shape[2]
    cap = table.shape[1] * page
    O, A, S = np.full(Q.shape, np.nan), np.full(Q.shape, np.nan), np.full(Q.shape, np.nan)
    G = Q.shape[1] // heads
    for b in range(len(positions)):
        n = int(offsets[b + 1]) - int(offsets[b])
        last = min(int(positions[b]) + n, cap)
        if n <= 0 or last <= 0:
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            K, V, ok = op.gather(arrays, table[b], last)
        t = np.arange(last)
        scales = np.abs(arrays[4].astype(np.float64))[np.where(ok, np.asarray(table[b])[t // page], 0), :, t % page]
        for i in range(n):
            p, row = int(positions[b]) + i, int(offsets[b]) + i
            if not 0 <= p < cap:
                continue
            t = np.arange(p + 1)
            use = np.nonzero(ok[:p + 1] & ((t > p - window) | (t < sinks)))[0]
            for hk in range(heads):
                rows = slice(hk * G, (hk + 1) * G)
                if not len(use):
                    O[row, rows] = A[row, rows] = S[row, rows] = 0.0
                    continue
                x = Q[row, rows] @ K[use, hk].T * float(scale)
                e = np.exp(x - x.max(1, keepdims=True))
                e /= e.sum(1, keepdims=True)
                O[row, rows], A[row, rows] = e @ V[use, hk], e @ np.abs(V[use, hk])
                S[row, rows] = (e @ scales[use, hk])[:, None]
    return O, A, S
