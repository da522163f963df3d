"""Performance cases of the paged cache and the rotary positions: what a server that keeps its sequences in pages does around
the products of a layer.

    listed()              the named cases
    draw(rng)             one more case of the same ranges (rng: random.Random)
    prepare(case, seed)   inputs, page pool and tables: what the program holds before the call
    run(state)            one pass: with `own` the library's entry points, without it their plain form
    work(case)            bytes and operations that one pass cannot do without
    exact(case, seed)     the same outputs from the definitions in 64 bits

Four kinds of work (case["kind"]):

    rope    rotary positions of packed tokens
    write   new tokens into the pages of a quantised cache, keys (and the queries beside them) rotated on the way, and what
            was stored read back: rotation, quantisation, storing, reading
    read    a cached prefix read back from its pages
    attn    attention of every sequence's new tokens over its pages: decoding steps, drafted tokens, chunks, whole prompts

Page pool: codes of `bits` bits in runs of 32 tokens x 128 dimensions in matrix-core operand order, [pages][kv_heads][page / 32]
runs for keys and as many for values, and fp16 (scale, zero-point) pairs [pages][kv_heads][page][key, value][scale, zero].
Queries, keys and values are Gaussian fp16.
"""
from __future__ import annotations

import math

import torch

own = False                      # True: the library's entry points instead of the plain form

HEAD = 128                       # head dimension of the cache
ROOT = HEAD ** -0.5              # softmax scale
DEV = "cuda"


def listed():
    return [
        # Sixteen sequences being generated: the queries' rotation on its own, the smallest call there is.
        {"name": "rope_16_tokens", "kind": "rope", "tokens": 16, "heads": 32, "dim": 128, "rot": 128, "layout": "half", "scaling": "none", "far": 8192},
        # A packed batch of long prompts: neighbouring pairs, half of the head, positions far beyond the trained length.
        {"name": "rope_8192_tokens_part", "kind": "rope", "tokens": 8192, "heads": 32, "dim": 128, "rot": 64, "layout": "interleaved", "scaling": "ramp", "far": 131072},
        # A decoding step of sixteen sequences: one token each, rotated and stored.
        {"name": "write_kv8_16_decode", "kind": "write", "bits": 8, "page": 64, "batch": 16, "count": 1, "past": 8192, "q_heads": 32, "kv_heads": 8,
         "rot": 128, "layout": "half", "scaling": "none"},
        # Ten prompts of different lengths that start inside a page, 4-bit codes, an odd group of query heads.
        {"name": "write_kv4_10_prompts", "kind": "write", "bits": 4, "page": 128, "batch": 10, "count": 901, "past": 77, "q_heads": 28, "kv_heads": 4,
         "rot": 64, "layout": "interleaved", "scaling": "wavelength"},
        # Two cached prefixes read back (to move them, or to attend over them elsewhere).
        {"name": "read_kv8_2x30000", "kind": "read", "bits": 8, "page": 256, "batch": 2, "context": 30000, "kv_heads": 8},
        # One sequence at an ordinary context: attention at its smallest.
        {"name": "attn_kv8_decode_1x2048", "kind": "attn", "bits": 8, "page": 64, "q_heads": 32, "kv_heads": 8,
         "decodes": 1, "context": 2048, "skew": False, "chunks": 0, "count": 0, "past": 0},
        # A full server: sequences of very different lengths, small pages, the 4-bit cache.
        {"name": "attn_kv4_decode_64_skewed", "kind": "attn", "bits": 4, "page": 32, "q_heads": 32, "kv_heads": 8,
         "decodes": 64, "context": 16384, "skew": True, "chunks": 0, "count": 0, "past": 0},
        # A few very long contexts of a large model.
        {"name": "attn_kv8_decode_4x60000", "kind": "attn", "bits": 8, "page": 256, "q_heads": 64, "kv_heads": 8,
         "decodes": 4, "context": 60000, "skew": False, "chunks": 0, "count": 0, "past": 0},
        # Drafted tokens being verified: five a sequence.
        {"name": "attn_kv8_verify_12x5", "kind": "attn", "bits": 8, "page": 64, "q_heads": 40, "kv_heads": 8,
         "decodes": 0, "context": 0, "skew": False, "chunks": 12, "count": 5, "past": 6000},
        # One chunk of a long prompt.
        {"name": "attn_kv4_chunk_512_after_30000", "kind": "attn", "bits": 4, "page": 128, "q_heads": 32, "kv_heads": 8,
         "decodes": 0, "context": 0, "skew": False, "chunks": 1, "count": 512, "past": 30000},
        # Decoding sequences and chunks of two prompts in one step.
        {"name": "attn_kv8_mixed_40_and_2", "kind": "attn", "bits": 8, "page": 64, "q_heads": 32, "kv_heads": 8,
         "decodes": 40, "context": 4000, "skew": False, "chunks": 2, "count": 1500, "past": 1000},
        # Whole prompts of different lengths, packed: the largest call.
        {"name": "attn_kv8_4_prompts_6000", "kind": "attn", "bits": 8, "page": 64, "q_heads": 32, "kv_heads": 8,
         "decodes": 0, "context": 0, "skew": False, "chunks": 4, "count": 6000, "past": 0},
    ]


MOST_PAIRS = 32 * (6000 * 3000 + 3 * 4500 * 2250)        # query heads x (row, token) pairs of the largest listed case
MOST_ROWS = 32 * 12000                                   # query heads x new tokens
MOST_TOKENS = 8 * 4 * 45000                              # KV heads x cached tokens read by a decoding step


def _log_int(rng, lo, hi):
    """A whole number of [lo, hi], even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_rope(rng):
    return {"rot": rng.choice([32, 64, 96, 128, 128]), "layout": rng.choice(["half", "interleaved"]),
            "scaling": rng.choice(["none", "linear", "base", "wavelength", "ramp"])}


def draw(rng):
    kind = rng.choice(["rope", "write", "write", "read", "attn", "attn", "attn", "attn", "attn", "attn"])
    if kind == "rope":
        case = {"kind": kind, "tokens": _log_int(rng, 1, 8192), "heads": rng.choice([1, 4, 8, 28, 32]), "dim": 128, **_draw_rope(rng),
                "far": _log_int(rng, 2048, 1 << 20)}
        if rng.random() < 0.3:                           # another head dimension than the cache's
            case["dim"] = rng.choice([64, 96, 256])
            case["rot"] = min(case["rot"], case["dim"])
            case["tokens"] = min(case["tokens"], 4096)
        return case
    kv_heads = rng.choice([1, 2, 4, 8, 8, 32])
    per_kv = rng.choice([1, 4, 5, 7, 8, 16]) if kv_heads < 32 else 1
    case = {"kind": kind, "bits": rng.choice([8, 4]), "page": rng.choice([32, 64, 128, 256]), "q_heads": kv_heads * per_kv, "kv_heads": kv_heads}
    if kind == "write":
        case["batch"] = _log_int(rng, 1, 128)
        case["count"] = rng.choice([1, _log_int(rng, 2, 8192)])
        case["count"] = max(1, min(case["count"], 300000 // (case["batch"] * (2 * kv_heads + case["q_heads"]))))
        return {**case, "past": _log_int(rng, 1, 8192), **_draw_rope(rng)}
    if kind == "read":
        batch = _log_int(rng, 1, 64)
        del case["q_heads"]
        return {**case, "batch": batch, "context": max(1, min(_log_int(rng, 16, 32768), 480000 // (batch * kv_heads)))}
    case |= {"decodes": 0, "context": 0, "skew": False, "chunks": 0, "count": 0, "past": 0}
    form = rng.choice(["decode", "decode", "verify", "chunk", "mixed", "prompt"])
    if form in ("decode", "mixed"):
        case["decodes"] = _log_int(rng, 1, 128)
        case["skew"] = rng.random() < 0.5
        case["context"] = min(_log_int(rng, 64, 65536), max(64, MOST_TOKENS // 2 // (case["decodes"] * kv_heads)))
    if form != "decode":
        case["chunks"] = {"verify": _log_int(rng, 1, 32), "chunk": rng.choice([1, 1, 2, 4]), "mixed": rng.choice([1, 2, 3]), "prompt": rng.choice([1, 2, 5, 8])}[form]
        case["count"] = _log_int(rng, 2, 16) if form == "verify" else _log_int(rng, 17, 4096)
        case["past"] = 0 if form == "prompt" else _log_int(rng, 16, 32768)
        while case["q_heads"] * case["chunks"] * case["count"] * (case["past"] + case["count"] / 2) > MOST_PAIRS / 2 or \
                kv_heads * case["chunks"] * (case["past"] + case["count"]) > MOST_TOKENS / 2 or \
                case["q_heads"] * case["chunks"] * case["count"] > MOST_ROWS:
            case["count"], case["past"] = max(2, case["count"] * 3 // 4), case["past"] * 3 // 4
    return case


# ------------------------------------------------------------------------------------------------ rotary frequencies

#: what the scaled forms take: factor, the length before it, and the bounds of the transition
SCALING = {"none": {}, "linear": {"factor": 4.0}, "base": {"factor": 8.0},
           "wavelength": {"factor": 8.0, "original_len": 8192, "low": 1.0, "high": 4.0},
           "ramp": {"factor": 16.0, "original_len": 8192, "low": 1.0, "high": 32.0}}
BASE = {"none": 10000.0, "linear": 10000.0, "base": 10000.0, "wavelength": 500000.0, "ramp": 10000.0}


def _frequencies(rot, scaling):
    """(radians per position of every pair, factor of the rotated values)."""
    p, base = SCALING[scaling], BASE[scaling]
    if scaling == "base":
        base *= p["factor"] ** (rot / (rot - 2))
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        f = [x / p["factor"] for x in f]
    if scaling == "wavelength":                          # short waves as they are, long ones stretched, a transition between
        share = [(p["original_len"] * x / (2 * math.pi) - p["low"]) / (p["high"] - p["low"]) for x in f]
        share = [min(1.0, max(0.0, s)) for s in share]
        f = [x * s + x / p["factor"] * (1 - s) for x, s in zip(f, share)]
    if scaling == "ramp":                                # the same with a transition that is linear in the pair's number
        at = lambda turns: rot * math.log(p["original_len"] / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(p["high"])), 0), min(math.ceil(at(p["low"])), rot - 1)
        ramp = [min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001))) for i in range(rot // 2)]
        f = [x / p["factor"] * r + x * (1 - r) for x, r in zip(f, ramp)]
        return f, 0.1 * math.log(p["factor"]) + 1.0
    return f, 1.0


def _rotate(x, positions, freq, amp, layout):
    """fp16 [tokens][heads][dim] -> the same, rotated.  In 64 bits: angles of far positions, and a value next to a code's border must
    not depend on the last bit of a sine."""
    half = freq.numel()
    angle = positions.double()[:, None] * freq
    cos, sin = (angle.cos() * amp)[:, None], (angle.sin() * amp)[:, None]
    head, rest = x[..., :2 * half].double(), x[..., 2 * half:]
    if layout == "half":
        a, b = head[..., :half], head[..., half:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((turned.float().half(), rest), -1)


# -------------------------------------------------------------------------------------------------------- page pool

NIBBLE = [0, 2, 4, 6, 1, 3, 5, 7]                        # operand element in nibble p of a word of 4-bit codes


def _quantise(x, bits):
    """fp16 [..., 128] -> (codes uint8 [..., 128], scale fp16 [...], zero-point fp16 [...])."""
    top = 2 ** bits - 1
    x = x.float()
    mn, mx = x.amin(-1), x.amax(-1)
    s = ((mx - mn) / top).half()
    s = torch.where((s > 0) & torch.isfinite(s), s, torch.ones_like(s))
    z = (-mn / s.float()).round().clamp(0, top)
    q = ((x / s.float()[..., None]).round() + z[..., None]).clamp(0, top)
    return q.to(torch.uint8), s, z.half()


def _views(pool):
    """The pool's code buffers with one axis per index of the operand order (and the bits of a code)."""
    k, v, pairs = pool
    pages, heads, page = pairs.shape[:3]
    lead = (pages, heads, page // 32)
    if k.shape[-1] == 4096:
        return k.view(*lead, 2, 2, 4, 16, 16), v.view(*lead, 4, 4, 16, 2, 2, 4), 8
    return k.view(*lead, 2, 4, 16, 4, 4), v.view(*lead, 2, 4, 16, 4, 4), 4


def _store(pool, page, at, K, V):
    """Keys and values fp16 [n][heads][128] into slot `at` of page `page` (both [n])."""
    kc, vc, bits = _views(pool)
    n, heads = K.shape[:2]
    run, u = at // 32, at % 32
    qk, sk, zk = _quantise(K, bits)
    qv, sv, zv = _quantise(V, bits)
    pool[2][page, :, at] = torch.stack((torch.stack((sk, zk), -1), torch.stack((sv, zv), -1)), -2)
    if bits == 8:
        kc[page, :, run, u // 16, :, :, u % 16, :] = qk.view(n, heads, 4, 2, 16).transpose(2, 3)
        vc[page, :, run, :, u % 16 // 4, :, :, u // 16, u % 4] = qv.view(n, heads, 4, 2, 16).transpose(3, 4)
        return
    nib = qk.view(n, heads, 4, 4, 8)[..., NIBBLE]
    kc[page, :, run, u // 16, :, u % 16] = nib[..., 0::2] | (nib[..., 1::2] << 4)
    # a byte of the value words holds two tokens: the low halves first, then the high ones
    e = u % 4 + u // 16 * 4
    p = e // 2 + e % 2 * 4
    qv = qv.view(n, heads, 2, 4, 16).transpose(3, 4)     # [n][heads][i / 4][c][i % 4]
    for high in (0, 1):
        pick = (p % 2 == high).nonzero()[:, 0] if n > 1 else torch.arange(n, device=DEV)
        where = (page[pick], slice(None), run[pick], slice(None), u[pick] % 16 // 4, slice(None), slice(None), p[pick] // 2)
        old, new = vc[where], qv[pick]
        if n > 1:
            vc[where] = (old & 0x0F | new << 4) if high else (old & 0xF0 | new)
        else:                                            # no selection that depends on data: one token
            vc[where] = torch.where((p % 2 == high)[:, None, None, None, None], (old & 0x0F | new << 4) if high else (old & 0xF0 | new), old)


def _load(pool, page, at):
    """(keys, values) fp32 [n][heads][128] from slot `at` of page `page`."""
    kc, vc, bits = _views(pool)
    n, heads = page.numel(), pool[2].shape[1]
    run, u = at // 32, at % 32
    if bits == 8:
        k = kc[page, :, run, u // 16, :, :, u % 16, :].transpose(2, 3).reshape(n, heads, HEAD)
        v = vc[page, :, run, :, u % 16 // 4, :, :, u // 16, u % 4].transpose(3, 4).reshape(n, heads, HEAD)
    else:
        b = kc[page, :, run, u // 16, :, u % 16]
        nib = torch.stack((b & 15, b >> 4), -1).flatten(-2)
        k = nib[..., [NIBBLE.index(e) for e in range(8)]].reshape(n, heads, HEAD)
        e = u % 4 + u // 16 * 4
        p = e // 2 + e % 2 * 4
        b = vc[page, :, run, :, u % 16 // 4, :, :, p // 2]
        v = (b >> (p % 2 * 4)[:, None, None, None, None] & 15).transpose(3, 4).reshape(n, heads, HEAD)
    pairs = pool[2][page, :, at].float()                 # [n][heads][key, value][scale, zero]
    return [(q.float() - pairs[:, :, i, 1, None]) * pairs[:, :, i, 0, None] for i, q in enumerate((k, v))]


# ----------------------------------------------------------------------------------------------------------- inputs

class _Inputs:
    """Everything random of a case, from one seed, on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        self.h = torch.Generator()
        self.h.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device=DEV).half()

    def shuffled(self, values):
        return [values[i] for i in torch.randperm(len(values), generator=self.h).tolist()]

    def pool(self, pages, heads, page, bits, filled=True):
        """A pool whose every slot has been stored once."""
        k = torch.zeros(pages, heads, page // 32, 512 * bits, dtype=torch.uint8, device=DEV)
        v, pairs = torch.zeros_like(k), torch.zeros(pages, heads, page, 2, 2, dtype=torch.float16, device=DEV)
        pool, step = (k, v, pairs), max(1, (1 << 27) // (heads * page * HEAD))
        for p0 in range(0, pages if filled else 0, step):
            n = min(step, pages - p0)
            at = torch.arange(page, device=DEV).repeat(n)
            where = torch.arange(p0, p0 + n, device=DEV).repeat_interleave(page)
            _store(pool, where, at, self.normal(n * page, heads, HEAD), self.normal(n * page, heads, HEAD))
        return pool

    def table(self, lens, page):
        """Pages of every sequence in no order, the rest of its row -1; (table, pages of the pool)."""
        need = [-(-n // page) for n in lens]
        ids = torch.randperm(sum(need) + 3, generator=self.h)
        rows = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
        done = 0
        for b, n in enumerate(need):
            rows[b, :n] = ids[done:done + n]
            done += n
        return rows.to(DEV), len(ids)


def _between(lo, hi, n):
    """n whole numbers from hi down to lo, evenly."""
    return [hi - (hi - lo) * i // max(n - 1, 1) for i in range(n)]


def _sequences(c):
    """(new tokens, cached tokens) of every sequence of a case: sizes go by the case, their order and all values by the seed."""
    if c["kind"] == "read":
        return [(n, 0) for n in _between((c["context"] + 1) // 2, c["context"], c["batch"])]
    if c["kind"] == "write":
        n, counts, past = c["batch"], _between((c["count"] + 1) // 2, c["count"], c["batch"]), _between(0, c["past"], c["batch"])
    else:
        # verification drafts as many tokens for every sequence; chunks and prompts are of different lengths
        n, lo = c["chunks"], c["count"] if c["count"] <= 16 else (c["count"] + 1) // 2
        counts, past = _between(lo, c["count"], n), _between((c["past"] + 1) // 2, c["past"], n)
    together = [(counts[i], past[i * 7 % n if n % 7 else i]) for i in range(n)]
    if c["kind"] == "attn" and c["decodes"]:
        m, top = c["decodes"], c["context"]
        lens = [max(1, int(top * (1 - i / m) ** 3)) for i in range(m)] if c["skew"] else _between((top + 1) // 2, top, m)
        together += [(1, n - 1) for n in lens]
    return together


def _batch(r, case):
    """Tables and positions of the case's sequences."""
    counts, past = map(list, zip(*r.shuffled(_sequences(case))))
    table, pages = r.table([n + p for n, p in zip(counts, past)], case["page"])
    offsets = torch.tensor([0] + counts).cumsum(0)
    seq = torch.arange(len(counts)).repeat_interleave(torch.tensor(counts))
    at = torch.arange(int(offsets[-1])) - offsets[seq] + torch.tensor(past)[seq]
    return {"counts": counts, "past": past, "table": table, "pages": pages, "offsets": offsets.int().to(DEV),
            "positions": torch.tensor(past, dtype=torch.int32, device=DEV), "seq": seq.to(DEV), "at": at.to(DEV)}


def _slots(s, page):
    """Page and slot of every new token."""
    return s["table"][s["seq"], s["at"] // page].long(), s["at"] % page


def prepare(case, seed):
    r, c = _Inputs(seed), case
    state = {"case": case, **globals()["_prepare_" + case["kind"]](case, r)}
    if c["kind"] in ("rope", "write"):
        f, state["amp"] = _frequencies(c["rot"], c["scaling"])
        state["freq"] = torch.tensor(f, dtype=torch.float64, device=DEV)
    if own:                                              # the handles that a program makes once
        import paper_2508_15601_amd as tm
        if c["kind"] in ("rope", "write"):
            kind = {"none": tm.TM_ROPE_PLAIN, "linear": tm.TM_ROPE_LINEAR, "base": tm.TM_ROPE_BASE, "wavelength": tm.TM_ROPE_WAVELENGTH, "ramp": tm.TM_ROPE_RAMP}
            state["rope"] = tm.tm_rope_create(c["rot"], layout=tm.TM_ROPE_HALF if c["layout"] == "half" else tm.TM_ROPE_INTERLEAVED,
                                              base=BASE[c["scaling"]], scaling=kind[c["scaling"]], **SCALING[c["scaling"]])
        if c["kind"] != "rope":
            state["cache"] = tm.tm_paged_create(*state["pool"])
            state["batch"] = tm.PagedBatch(state["table"], state["offsets"], state["positions"], max_count=max(state["counts"]),
                                           max_len=max(n + p for n, p in zip(state["counts"], state["past"])))
    return state


def run(state):
    return globals()["_own_" + state["case"]["kind"] if own else "_plain_" + state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------------------- rope

def _prepare_rope(c, r):
    x = r.normal(c["tokens"], c["heads"], c["dim"])
    at = torch.randint(0, c["far"], (c["tokens"],), generator=r.g, device=DEV, dtype=torch.int32)
    return {"X": x, "positions": at, "Y": torch.empty_like(x)}


def _plain_rope(s):
    return _rotate(s["X"], s["positions"], s["freq"], s["amp"], s["case"]["layout"])


def _own_rope(s):
    import paper_2508_15601_amd as tm
    return tm.tm_rope_apply(s["X"], s["positions"], s["rope"], s["Y"])


# ------------------------------------------------------------------------------------------------------------ write

def _prepare_write(c, r):
    Hq, Hk = c["q_heads"], c["kv_heads"]
    s = _batch(r, c)
    n = sum(s["counts"])
    qkv = r.normal(n, Hq + 2 * Hk, HEAD)                 # what the fused projection left: keys and values lie behind the queries
    q, k, v = qkv.split((Hq, Hk, Hk), 1)
    new = lambda heads: torch.empty(n, heads, HEAD, dtype=torch.float16, device=DEV)  # noqa: E731
    return {**s, "pool": r.pool(s["pages"], Hk, c["page"], c["bits"], filled=False), "Q": q, "K": k, "V": v,
            "rotated": new(Hq), "K_back": new(Hk), "V_back": new(Hk)}


def _plain_write(s):
    c = s["case"]
    q, k = (_rotate(x, s["at"], s["freq"], s["amp"], c["layout"]) for x in (s["Q"], s["K"]))
    page, slot = _slots(s, c["page"])
    _store(s["pool"], page, slot, k, s["V"])
    k, v = _load(s["pool"], page, slot)
    return q, k.half(), v.half()


def _own_write(s):
    import paper_2508_15601_amd as tm
    tm.tm_paged_append(s["cache"], s["batch"], s["K"], s["V"], rope=s["rope"], Q=s["Q"], Q_out=s["rotated"])
    tm.tm_paged_read(s["cache"], s["batch"], s["K_back"], s["V_back"])
    return s["rotated"], s["K_back"], s["V_back"]


# ------------------------------------------------------------------------------------------------------------- read

def _prepare_read(c, r):
    s = _batch(r, c)
    new = lambda: torch.empty(sum(s["counts"]), c["kv_heads"], HEAD, dtype=torch.float16, device=DEV)  # noqa: E731
    return {**s, "pool": r.pool(s["pages"], c["kv_heads"], c["page"], c["bits"]), "K_back": new(), "V_back": new()}


def _plain_read(s):
    k, v = _load(s["pool"], *_slots(s, s["case"]["page"]))
    return k.half(), v.half()


def _own_read(s):
    import paper_2508_15601_amd as tm
    tm.tm_paged_read(s["cache"], s["batch"], s["K_back"], s["V_back"])
    return s["K_back"], s["V_back"]


# ------------------------------------------------------------------------------------------------------------- attn

def _prepare_attn(c, r):
    s = _batch(r, c)
    q = r.normal(sum(s["counts"]), c["q_heads"], HEAD)
    return {**s, "pool": r.pool(s["pages"], c["kv_heads"], c["page"], c["bits"]), "Q": q, "O": torch.empty_like(q)}


def _plain_attn(s):
    """Sequences with as many new tokens go together, padded to the longest of them."""
    c, out = s["case"], torch.empty_like(s["O"])
    Hk, G = c["kv_heads"], c["q_heads"] // c["kv_heads"]
    for n in sorted(set(s["counts"])):
        same = [b for b, m in enumerate(s["counts"]) if m == n]
        past = s["positions"][same].long()
        longest = max(s["past"][b] for b in same) + n
        t = torch.arange(longest, device=DEV)
        page = s["table"][same][:, t // c["page"]].clamp_min(0).long()                   # behind a sequence: masked
        k, v = _load(s["pool"], page.flatten(), (t % c["page"]).repeat(len(same)))
        k, v = (x.view(len(same), longest, Hk, HEAD).transpose(1, 2).contiguous() for x in (k, v))
        rows = s["offsets"][same].long()[:, None] + torch.arange(n, device=DEV)
        q = s["Q"][rows].float().view(len(same), n, Hk, G, HEAD).permute(0, 2, 1, 3, 4).reshape(len(same), Hk, n * G, HEAD)
        x = torch.matmul(q, k.transpose(2, 3)).mul_(ROOT).view(len(same), Hk, n, G, longest)
        seen = t <= past[:, None, None] + torch.arange(n, device=DEV)[:, None]           # [sequences][n][tokens]
        x = x.masked_fill_(~seen[:, None, :, None], -math.inf)
        x = (x - x.amax(-1, keepdim=True)).exp_()
        x = x.div_(x.sum(-1, keepdim=True)).view(len(same), Hk, n * G, longest)
        o = torch.matmul(x, v).view(len(same), Hk, n, G, HEAD).permute(0, 2, 1, 3, 4)
        out[rows] = o.reshape(len(same), n, c["q_heads"], HEAD).half()
    return out


def _own_attn(s):
    import paper_2508_15601_amd as tm
    return tm.tm_paged_attn(s["Q"], s["cache"], s["batch"], s["O"], ROOT)


# ----------------------------------------------------------------------------------------------------- work, exact

def _token_bytes(bits):
    """Codes and pairs of one token and KV head, key and value."""
    return 2 * HEAD * bits // 8 + 8


def work(case):
    c, kind = case, case["kind"]
    if kind == "rope":
        return {"bytes": c["tokens"] * (4 * c["heads"] * c["dim"] + 4), "flops": 3.0 * c["tokens"] * c["heads"] * c["rot"]}
    seqs = _sequences(c)
    n = sum(m for m, _ in seqs)
    if kind == "read":
        return {"bytes": n * c["kv_heads"] * (_token_bytes(c["bits"]) + 4 * HEAD), "flops": 4.0 * n * c["kv_heads"] * HEAD}
    if kind == "write":
        moved = c["kv_heads"] * (2 * _token_bytes(c["bits"]) + 8 * HEAD) + 4 * c["q_heads"] * HEAD
        return {"bytes": n * moved, "flops": n * HEAD * (13.0 * c["kv_heads"] + 3.0 * c["q_heads"])}
    pairs = sum(m * past + m * (m + 1) / 2 for m, past in seqs)              # (row, token it attends over)
    return {"bytes": sum(m + past for m, past in seqs) * c["kv_heads"] * _token_bytes(c["bits"]) + 4 * n * c["q_heads"] * HEAD,
            "flops": 4.0 * HEAD * c["q_heads"] * pairs}


def _stored64(x, bits):
    """What a quantised cache holds for the vectors x (64 bits): scale to fp16, codes to the nearest."""
    top = 2 ** bits - 1
    lo, hi = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
    scale = ((hi - lo) / top).float().half().double()
    scale[scale == 0] = 1.0
    zero = torch.clamp(torch.round(-lo / scale), 0, top)
    return (torch.clamp(torch.round(x / scale) + zero, 0, top) - zero) * scale


def _turned64(x, at, c):
    """Rotation as a product of complex numbers; x fp16 [n][heads][dim]."""
    f, amp = _frequencies(c["rot"], c["scaling"])
    turn = torch.polar(torch.full((1, 1), amp, dtype=torch.float64, device=DEV), at.double()[:, None] * torch.tensor(f, dtype=torch.float64, device=DEV))[:, None]
    x, y = x.double(), x.double().clone()
    first, second = (slice(0, c["rot"] // 2), slice(c["rot"] // 2, c["rot"])) if c["layout"] == "half" else (slice(0, c["rot"], 2), slice(1, c["rot"], 2))
    z = torch.complex(x[..., first], x[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "rope":
        return _turned64(s["X"], s["positions"], c)
    if c["kind"] == "write":
        keys = _turned64(s["K"], s["at"], c).float().half().double()                     # a key is stored from its fp16 value
        return _turned64(s["Q"], s["at"], c), _stored64(keys, c["bits"]), _stored64(s["V"].double(), c["bits"])
    page, kv = c["page"], []
    for b in range(len(s["counts"])):                    # codes of every sequence, token by token, from the layout's index formulas
        t = torch.arange(s["past"][b] + s["counts"][b], device=DEV)
        kv.append(_codes64(s["pool"], s["table"][b, t // page].long(), t % page))
    if c["kind"] == "read":
        return torch.cat([k for k, _ in kv]), torch.cat([v for _, v in kv])
    out, row = [], 0
    for b, n in enumerate(s["counts"]):
        k, v = (x.transpose(0, 1).repeat_interleave(c["q_heads"] // c["kv_heads"], 0) if n <= 16 else x for x in kv[b])
        mask = torch.arange(s["past"][b] + n, device=DEV) > s["past"][b] + torch.arange(n, device=DEV)[:, None]
        q, heads = s["Q"][row:row + n].double().transpose(0, 1), []
        for h in range(c["q_heads"]) if n > 16 else [slice(None)]:                       # a long chunk one head at a time
            kh, vh = (k, v) if n <= 16 else (x[:, h // (c["q_heads"] // c["kv_heads"])] for x in (k, v))
            logits = torch.where(mask, -math.inf, q[h] @ kh.transpose(-1, -2) / math.sqrt(HEAD))
            heads.append(torch.softmax(logits, -1) @ vh)
        out.append((heads[0] if n <= 16 else torch.stack(heads)).transpose(0, 1))
        row += n
    return torch.cat(out)


def _codes64(pool, page, at):
    """Keys and values [n][heads][128] in 64 bits: every code by its address in the pool."""
    k, v, pairs = pool
    bits, heads, runs = k.shape[-1] // 512, k.shape[1], k.shape[2]
    d, u = torch.arange(HEAD, device=DEV), (at % 32)[:, None]
    run = ((page[:, None] * heads + torch.arange(heads, device=DEV)) * runs + (at // 32)[:, None])[:, :, None]
    i, hh, e = d // 16, u % 16 // 4, u % 4 + u // 16 * 4
    if bits == 8:
        to_k = (u // 16 * 2 + d % 32 // 16) * 1024 + (16 * (d // 32) + u % 16) * 16 + d % 16
        to_v = (i // 2 * 64 + 16 * hh + d % 16) * 16 + i % 2 * 8 + e
        codes = k.flatten()[run * 4096 + to_k[:, None]], v.flatten()[run * 4096 + to_v[:, None]]
    else:
        nib = lambda element: element // 2 + element % 2 * 4  # noqa: E731
        to_k = ((u // 16 * 64 + 16 * (d // 32) + u % 16) * 4 + d % 32 // 8) * 8 + nib(d % 8)
        to_v = ((i // 4 * 64 + 16 * hh + d % 16) * 4 + i % 4) * 8 + nib(e)
        codes = [x.flatten()[run * 2048 + to[:, None] // 2] >> to[:, None] % 2 * 4 & 15 for x, to in ((k, to_k), (v, to_v))]
    pair = pairs[page, :, at].double()
    return [(q.double() - pair[:, :, j, 1:]) * pair[:, :, j, :1] for j, q in enumerate(codes)]
