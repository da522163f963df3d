"""GPU parity of norms of heads where a wave takes many heads, a round after the other: the next heads are requested while these are worked on, weights are loaded anew where heads have their own, and
the last round may be partial.  Bit for bit against calls of few tokens, whose waves take a round each, and some rows against the 64-bit oracle with the tolerance of test_gpu_heads.py."""
import sys

import numpy as np
import pytest

from test_gpu_heads import Heads, Pool, _dev, _host, _near, tm  # noqa: F401

pytestmark = pytest.mark.gpu


def _check_rows(s, outs, rows):
    for side, got in outs:
        want, size = s.want(side, rows)
        assert _near(_host(got[rows]), want, size).all()


@pytest.mark.parametrize("tokens, q_heads, k_heads, dim, rot, layout, axes, norm, centred, without", [
    # rounds of a token: all of a wave's number (5), fewer, queries and keys in one wave, partial last ones
    (1500, 64, 4, 128, 128, "half", 1, "shared", False, ""),
    (1500, 64, 4, 128, 64, "interleaved", 3, "own", True, ""),
    (1230, 75, 5, 128, 128, "half", 2, "own", False, ""),
    (2600, 33, 3, 128, 96, "half", 1, "shared", True, ""),
    (2600, 28, 4, 128, 128, "interleaved", 1, "own", False, "Q"),          # one side normed
    (2600, 28, 4, 128, 128, "half", 1, "shared", True, "K"),
    (5000, 30, 17, 64, 64, "half", 2, "own", False, ""),                  # sixteen heads at a time
    (2100, 21, 6, 256, 128, "half", 1, "own", True, ""),                  # four
    (14000, 40, 8, 24, 16, "interleaved", 1, "shared", False, ""),
    (1500, 64, 4, 128, 128, "half", 1, "none", False, ""),
])
def test_rounds_of_a_wave(tm, tokens, q_heads, k_heads, dim, rot, layout, axes, norm, centred, without):  # noqa: F811
    import torch
    print(f"heads tokens={tokens} {q_heads}/{k_heads} dim={dim} rot={rot} {layout} {norm} without={without}", file=sys.stderr, flush=True)
    lanes = 1 << max(0, -(-dim // 16) - 1).bit_length()
    rounds = -(-q_heads * lanes // 64) - (-k_heads * lanes // 64)
    assert tokens * rounds >= 12288 and tokens * q_heads * k_heads * dim < 1 << 31
    s = Heads(tm, tokens, q_heads, k_heads, dim, rot, layout, axes, norm, 0.25, centred)
    for side in without:
        s.norm[side] = None
    Q, K = torch.full_like(s.X["Q"], 7.0).contiguous(), torch.full_like(s.X["K"], 7.0).contiguous()
    s.apply(Q, K)
    _check_rows(s, (("Q", Q), ("K", K)), np.r_[0:3, tokens // 2, tokens - 2:tokens])
    for t in range(0, tokens, 200):                                        # fewer than 6144 rounds: one to a wave
        part = slice(t, min(t + 200, tokens))
        q, k = torch.empty_like(Q[part]), torch.empty_like(K[part])
        tm.tm_heads_apply(rope=s.rope, positions=s.positions[part].contiguous(), Q=s.X["Q"][part], Q_out=q, q_norm=s.norm["Q"], K=s.X["K"][part], K_out=k, k_norm=s.norm["K"])
        assert torch.equal(q, Q[part]) and torch.equal(k, K[part])
    s.apply(s.X["Q"], s.X["K"])                                            # in place
    assert torch.equal(s.X["Q"], Q) and torch.equal(s.X["K"], K)


@pytest.mark.parametrize("bits, counts, past, q_heads, heads, rot, layout, axes, norm, centred, without", [
    # from 131072 query vectors on a wave takes all of a token's: 28 heads are four rounds, 33 five, the last one partial
    (8, [2300, 1, 2400], [0, 90, 31], 28, 4, 128, "half", 1, "shared", False, ""),
    (4, [2300, 1, 2400], [0, 90, 31], 28, 4, 128, "half", 3, "own", True, ""),
    (4, [1990, 2000], [5, 0], 33, 3, 64, "interleaved", 1, "own", False, ""),
    (8, [1990, 2000], [5, 0], 33, 3, 128, "interleaved", 1, "shared", True, ""),
    (8, [4700], [17], 28, 4, 96, "half", 2, "own", True, "K"),             # one side normed
    (4, [4700], [17], 28, 4, 128, "half", 1, "shared", False, "Q"),
    (8, [4700], [17], 28, 4, 128, "interleaved", 1, "own", True, "Q"),
    (8, [1990, 2000], [5, 0], 33, 3, 0, "half", 1, "own", False, ""),      # not turned
])
def test_rounds_of_a_wave_in_the_append(tm, bits, counts, past, q_heads, heads, rot, layout, axes, norm, centred, without):  # noqa: F811
    import torch
    print(f"append bits={bits} counts={counts} {q_heads}/{heads} rot={rot} {layout} axes={axes} {norm} without={without}", file=sys.stderr, flush=True)
    a, b = (Pool(tm, bits, 64, heads, counts, past, seed=5) for _ in range(2))
    assert a.tokens * q_heads >= 16384 * 8 and q_heads > 8
    s = Heads(tm, a.tokens, q_heads, heads, 128, rot, layout, axes, norm, 0.25, centred)
    for side in without:
        s.norm[side] = None
    own = axes == 1 and rot                                               # turned by the sequences' positions
    if own:
        s.pos, s.positions = a.at[:, None], _dev(a.at.astype(np.int32))
    V = torch.randn(a.tokens, heads, 128, device="cuda").half()
    Q, K = torch.empty(a.tokens, q_heads, 128, dtype=torch.float16, device="cuda"), torch.empty(a.tokens, heads, 128, dtype=torch.float16, device="cuda")
    s.apply(Q, K)
    _check_rows(s, (("Q", Q), ("K", K)), np.r_[1:3, a.tokens // 2, a.tokens - 4:a.tokens - 2])
    tm.tm_paged_append(a.cache, a.batch, K, V)
    out = torch.full((a.tokens, q_heads + 1, 128), 7.0, dtype=torch.float16, device="cuda")
    args = dict(rope=s.rope, q_norm=s.norm["Q"], k_norm=s.norm["K"], positions=None if own else s.positions)
    tm.tm_paged_append(b.cache, b.batch, s.X["K"], V, Q=s.X["Q"], Q_out=out[:, 1:], **args)
    for x, y in zip(a.contents(), b.contents()):
        assert torch.equal(x, y)
    assert torch.equal(out[1:-2, 1:], Q[1:-2]) and (out[:, 0] == 7).all() and (out[[0, -2, -1]] == 7).all()
    tm.tm_paged_append(b.cache, b.batch, s.X["K"], V, Q=s.X["Q"], Q_out=s.X["Q"], **args)      # in place
    assert torch.equal(s.X["Q"][1:-2], Q[1:-2])
