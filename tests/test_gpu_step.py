"""A server's steps as they would be run: pages from lengths, norms and rotation on the way into the cache, attention in a window, pages behind the window and behind refused drafts given
back - against a history of every row's tokens kept on the host."""
import numpy as np
import pytest

from oracle import oracle_attn as oa
from oracle import oracle_step as st

pytestmark = pytest.mark.gpu

WINDOW, SINKS, PAGE, HEADS, Q_HEADS, SCALE = 70, 5, 32, 2, 8, 128 ** -0.5
# new tokens of the rows at every step, and how many of them are refused afterwards
STEPS = [([40, 0, 130, 1], None), ([1, 33, 1, 1], None), ([5, 5, 5, 5], [3, 0, 4, 5]), ([1, 1, 1, 1], None), ([64, 1, 0, 1], None), ([1, 90, 1, 200], None), ([1, 1, 1, 1], [1, 0, 1, 0])]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("hints", [False, True])
def test_steps_of_a_server(bits, hints):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_2508_15601_amd as tm
    g = torch.Generator(device="cuda")
    g.manual_seed(bits)
    rows, pages, max_pages = 4, 40, 20
    cache = tm.tm_paged_create(*tm.tm_paged_pool(pages, HEADS, PAGE, bits))
    for t in (cache.k, cache.v):
        t.random_(0, 256, generator=g)
    cache.pairs.view(torch.int16).random_(-32768, 32767, generator=g)
    free = tm.tm_page_list(pages)
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    table, lens = torch.full((rows, max_pages), -1, dtype=torch.int32, device="cuda"), ints(rows)
    batch = tm.PagedBatch(table, ints(rows + 1), ints(rows))
    rope = tm.tm_rope_create(64, axis=[i % 3 for i in range(32)])
    norms = [tm.HeadNorm(1 + 0.2 * torch.randn(128, generator=g, device="cuda").half(), offset=0.5) for _ in range(2)]
    K_hist, V_hist = ([np.zeros((0, HEADS, 128)) for _ in range(rows)] for _ in range(2))
    behind = ints(rows)
    for step, (counts, refused) in enumerate(STEPS):
        print(f"step {step}: {counts} refused {refused}", flush=True)
        n = sum(counts)
        qkv = torch.randn(n, Q_HEADS + 2 * HEADS, 128, generator=g, device="cuda").half()
        q, k, v = qkv.split((Q_HEADS, HEADS, HEADS), 1)
        places = torch.randint(0, 5000, (n, 3), generator=g, device="cuda", dtype=torch.int32)
        new, slots = torch.tensor(counts, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int64, device="cuda")
        if hints:
            batch.max_count, batch.max_len = max(counts), max(len(h) for h in K_hist) + max(counts)
        tm.tm_paged_assign(cache, free, batch, lens, new, slots=slots)
        Q, O = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty(n, Q_HEADS, 128, dtype=torch.float16, device="cuda")
        tm.tm_paged_append(cache, batch, k, v, rope=rope, Q=q, Q_out=Q, q_norm=norms[0], k_norm=norms[1], positions=places)
        tm.tm_paged_attn(Q, cache, batch, O, SCALE, window=WINDOW, sinks=SINKS)
        # the same tokens on the host: keys from the pass over heads alone, codes by the oracle
        K = torch.empty_like(k, memory_format=torch.contiguous_format)
        tm.tm_heads_apply(rope=rope, positions=places, K=k, K_out=K, k_norm=norms[1])
        torch.cuda.synchronize()
        kh, vh = (oa.kv_dequant(*oa.kv_quantise(x.cpu().numpy(), bits)) for x in (K, v.contiguous()))
        got, Qh, at = O.cpu().numpy().astype(np.float64), Q.cpu().numpy().astype(np.float64), 0
        for b, c in enumerate(counts):
            past = len(K_hist[b])
            K_hist[b], V_hist[b] = np.concatenate([K_hist[b], kh[at:at + c]]), np.concatenate([V_hist[b], vh[at:at + c]])
            for i in range(c):
                seen = st.seen(past + i, WINDOW, SINKS)
                for h in range(Q_HEADS):
                    x = K_hist[b][seen, h // 4] @ Qh[at + i, h] * SCALE
                    e = np.exp(x - x.max())
                    e /= e.sum()
                    want, size = e @ V_hist[b][seen, h // 4], e @ np.abs(V_hist[b][seen, h // 4])
                    # as test_gpu_paged_attn.py has it; scales here are at most 8 / 15 (4-bit) or 8 / 255 for values up to 4
                    sums = 2.0 ** -24 * (10 * 1039 * 8 / 15 if bits == 4 else 25 * 1151 * 8 / 255)
                    assert (np.abs(got[at + i, h] - want) <= 1.125 * 2.0 ** -11 * (np.abs(want) + size) + 2.0 ** -25 + sums).all(), (step, b, i, h)
            at += c
        # what was refused leaves, and what no later token sees
        if refused is not None:
            lens.sub_(torch.tensor(refused, dtype=torch.int32, device="cuda"))
            tm.tm_paged_release(cache, free, table, first=lens)
            K_hist, V_hist = ([h[:len(h) - r] for h, r in zip(x, refused)] for x in (K_hist, V_hist))
        torch.sub(lens, WINDOW - 1, out=behind)
        tm.tm_paged_release(cache, free, table, first=torch.full_like(lens, SINKS), last=behind)
        torch.cuda.synchronize()
        held = table[table >= 0].tolist()
        left = free.pages[:int(free.count)].tolist()
        assert sorted(held + left) == list(range(pages))                  # every page is somewhere, once
        assert lens.tolist() == [len(h) for h in K_hist]
    assert max(len(h) for h in K_hist) > 200 and len(held) < 24           # the rows have outgrown what they hold
