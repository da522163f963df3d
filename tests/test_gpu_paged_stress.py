"""Repeat-determinism of the hand-overs of attention over pages at full size, as in test_gpu_stress.py: pieces of contexts that CTAs share, in one level and in two, pieces that single waves
share, both beside row tiles of the same launch, and the pieces of row tiles.  Every launch is followed by work that sweeps the L2s, and its output must equal the first one's bit for bit."""
import numpy as np
import pytest

from test_gpu_stress import _repeat, _say, env  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("name, counts, lengths, page, form", [
    ("one context in more than sixteen pieces", [1], [32768], 64, (1, 256, False)),
    ("four contexts", [1] * 4, [8192, 5000, 3000, 7000], 64, (1, 256, False)),
    ("drafts, two tiles a CTA", [5] * 12, [3000 + 250 * i for i in range(12)], 64, (1, 256, False)),
    ("every wave by itself", [1] * 130, [max(1, int(9000 * (1 - i / 130) ** 3)) for i in range(130)], 32, (1, 256, True)),
    ("decoding beside chunks", [1] * 40 + [1500, 750], [2000 + 50 * i for i in range(40)] + [2500, 1250], 64, (2, 128, True)),
    ("a chunk after a long past", [512], [30512], 128, (2, 0, False)),
])
def test_pieces_repeat_bit_for_bit(env, bits, name, counts, lengths, page, form):  # noqa: F811
    torch, tm, thrash = env
    heads, q_heads = 8, 32
    _say(f"stress paged attention {name}, KV{bits}")
    B = len(counts)
    need = [-(-n // page) for n in lengths]
    pages = sum(need)
    ids = np.random.default_rng(bits).permutation(pages).astype(np.int32)
    table, at = np.full((B, max(need)), -1, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    g = torch.Generator(device="cuda")
    g.manual_seed(bits)
    k, v = (torch.randint(0, 256, (pages, heads, page // 32, 512 * bits), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
    pairs = torch.empty(pages, heads, page, 2, 2, dtype=torch.float16, device="cuda")
    pairs[..., 0].uniform_(0.005, 0.05, generator=g)
    pairs[..., 1] = torch.randint(0, 1 << bits, pairs.shape[:-1], generator=g, device="cuda").half()
    cache = tm.tm_paged_create(k, v, pairs)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = tm.PagedBatch(dev(table), dev(np.cumsum([0] + counts)), dev([n - c for n, c in zip(lengths, counts)]), max_count=max(counts), max_len=max(lengths))
    tokens = sum(counts)
    assert tm.tm_get_paged_form(cache, batch, tokens, q_heads) == form
    Q = torch.randn(tokens, q_heads, 128, generator=g, device="cuda").half()
    O = torch.empty_like(Q)
    _repeat(torch, lambda: tm.tm_paged_attn(Q, cache, batch, O, 128 ** -0.5), O, thrash, f"{name}, KV{bits}")
    assert not torch.isnan(O).any()
    cache.close()
