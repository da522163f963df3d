"""Performance cases of the operators around a paged cache that a server's step takes besides storing and plain attention: pages for
the new tokens, norms of heads with the rotation, positions of several axes, attention in a sliding window.

    listed()              the named cases
    draw(rng)             one more case of the same ranges (rng: random.Random)
    prepare(case, seed)   inputs, page pool and tables: what the program holds before the call
    run(state)            one pass: with `own` the library's entry points, without it their plain form
    work(case)            bytes and operations that one pass cannot do without
    exact(case, seed)     the same outputs from the definitions in 64 bits

Four kinds of work (case["kind"]):

    heads    queries and keys of packed tokens normed head by head and turned for their positions, which have one axis or several
             (time, height and width of images and video)
    store    the same on the way into the pages of a quantised cache, and what was stored read back
    pages    pages of a free list given to the rows of a table by their lengths: tables, offsets, positions, slots of new tokens
    window   attention of every sequence's new tokens over its pages where a token sees the last `window` tokens and the first `sinks`

Page pool: codes of `bits` bits in runs of 32 tokens x 128 dimensions in matrix-core operand order, [pages][kv_heads][page / 32]
runs for keys and as many for values, and fp16 (scale, zero-point) pairs [pages][kv_heads][page][key, value][scale, zero].
"""
from __future__ import annotations

import math

import torch

own = False                      # True: the library's entry points instead of the plain form

HEAD = 128                       # head dimension of the cache
ROOT = HEAD ** -0.5              # softmax scale
EPS = 1e-6                       # of the norms
DEV = "cuda"


def listed():
    return [
        # Sixteen sequences being generated: the smallest call there is.
        {"name": "heads_16_tokens", "kind": "heads", "tokens": 16, "q_heads": 32, "k_heads": 8, "dim": 128, "norm": "shared", "offset": 0.0, "centred": False,
         "rot": 128, "layout": "half", "scaling": "none", "axes": 1, "far": 8192},
        # A packed batch of long prompts.
        {"name": "heads_8192_tokens", "kind": "heads", "tokens": 8192, "q_heads": 32, "k_heads": 8, "dim": 128, "norm": "shared", "offset": 1.0, "centred": False,
         "rot": 128, "layout": "half", "scaling": "ramp", "axes": 1, "far": 131072},
        # Weights of every head's own, the mean taken out, half of a head turned by neighbouring pairs.
        {"name": "heads_1500_tokens_own_weights", "kind": "heads", "tokens": 1500, "q_heads": 28, "k_heads": 4, "dim": 128, "norm": "own", "offset": 0.0, "centred": True,
         "rot": 64, "layout": "interleaved", "scaling": "none", "axes": 1, "far": 32768},
        # Patches of a picture in an image encoder: rows and columns are the axes, no norms, another head dimension than the cache's.
        {"name": "heads_4097_patches_2_axes", "kind": "heads", "tokens": 4097, "q_heads": 16, "k_heads": 16, "dim": 80, "norm": "none", "offset": 0.0, "centred": False,
         "rot": 80, "layout": "half", "scaling": "none", "axes": 2, "far": 64},
        # A decoding step of sixty-four sequences.
        {"name": "store_kv8_64_decode", "kind": "store", "bits": 8, "page": 64, "batch": 64, "count": 1, "past": 8192, "q_heads": 32, "kv_heads": 8,
         "norm": "shared", "offset": 0.0, "centred": False, "rot": 128, "layout": "half", "scaling": "none", "axes": 1},
        # Prompts with frames of a video in them: time, height and width.
        {"name": "store_kv4_6_prompts_3_axes", "kind": "store", "bits": 4, "page": 128, "batch": 6, "count": 1601, "past": 77, "q_heads": 28, "kv_heads": 4,
         "norm": "shared", "offset": 0.0, "centred": False, "rot": 128, "layout": "half", "scaling": "none", "axes": 3},
        # A decoding step of a full server: now and then a sequence needs another page.
        {"name": "pages_256_decode", "kind": "pages", "page": 64, "batch": 256, "count": 1, "past": 16384, "idle": 0.1, "scarce": False},
        # Prompts beside decoding sequences, and not pages for all of them.
        {"name": "pages_1000_with_prompts", "kind": "pages", "page": 32, "batch": 1000, "count": 900, "past": 9000, "idle": 0.6, "scarce": True},
        # One long sequence: attention at its smallest.
        {"name": "window_kv8_1024_decode_1x30000", "kind": "window", "bits": 8, "page": 64, "q_heads": 32, "kv_heads": 8, "window": 1024, "sinks": 0,
         "decodes": 1, "context": 30000, "skew": False, "chunks": 0, "count": 0, "past": 0},
        # A full server, the first tokens kept in sight.
        {"name": "window_kv8_4096_decode_64x20000", "kind": "window", "bits": 8, "page": 64, "q_heads": 32, "kv_heads": 8, "window": 4096, "sinks": 4,
         "decodes": 64, "context": 20000, "skew": False, "chunks": 0, "count": 0, "past": 0},
        # Decoding sequences of very different lengths and chunks of two long prompts in one step.
        {"name": "window_kv4_2048_mixed_24_and_2", "kind": "window", "bits": 4, "page": 32, "q_heads": 32, "kv_heads": 8, "window": 2048, "sinks": 64,
         "decodes": 24, "context": 20000, "skew": True, "chunks": 2, "count": 1024, "past": 12000},
        # Whole prompts of different lengths, packed: the largest call.
        {"name": "window_kv8_1024_4_prompts_6000", "kind": "window", "bits": 8, "page": 64, "q_heads": 32, "kv_heads": 8, "window": 1024, "sinks": 4,
         "decodes": 0, "context": 0, "skew": False, "chunks": 4, "count": 6000, "past": 0},
    ]


MOST_VALUES = 8192 * 40 * 128                            # values normed and turned in a call
MOST_SCORES = 32 * 2 * 1024 * 13000                      # query heads x rows x tokens that the plain form of a window works on


def _log_int(rng, lo, hi):
    """A whole number of [lo, hi], even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_turns(rng):
    return {"norm": rng.choice(["shared", "shared", "own", "none"]), "offset": rng.choice([0.0, 1.0]), "centred": rng.random() < 0.3,
            "rot": rng.choice([32, 64, 96, 128, 128]), "layout": rng.choice(["half", "interleaved"]),
            "scaling": rng.choice(["none", "linear", "base", "wavelength", "ramp"]), "axes": rng.choice([1, 1, 2, 3])}


def draw(rng):
    kind = rng.choice(["heads", "heads", "heads", "store", "store", "pages", "pages", "window", "window", "window", "window", "window"])
    if kind == "pages":
        batch = _log_int(rng, 1, 2048)
        case = {"kind": kind, "page": rng.choice([32, 64, 128, 256]), "batch": batch, "count": rng.choice([1, 5, _log_int(rng, 2, 8192)]), "past": _log_int(rng, 1, 32768),
                "idle": rng.choice([0.0, 0.3, 0.7]), "scarce": rng.random() < 0.3}
        case["count"] = max(1, min(case["count"], 1000000 // batch))
        case["past"] = max(1, min(case["past"], 16000000 // batch))
        return case
    if kind == "heads":
        q_heads, k_heads = rng.choice([(32, 8), (28, 4), (40, 8), (16, 16), (8, 1), (5, 5), (64, 4)])
        case = {"kind": kind, "tokens": 0, "q_heads": q_heads, "k_heads": k_heads, "dim": rng.choice([128, 128, 128, 64, 80, 96, 256]), **_draw_turns(rng),
                "far": _log_int(rng, 2048, 1 << 20)}
        case["rot"] = min(case["rot"], case["dim"])
        case["tokens"] = _log_int(rng, 1, MOST_VALUES // (case["dim"] * (q_heads + k_heads)))
        return case
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    per_kv = rng.choice([1, 4, 5, 7, 8])
    case = {"kind": kind, "bits": rng.choice([8, 4]), "page": rng.choice([32, 64, 128, 256]), "q_heads": kv_heads * per_kv, "kv_heads": kv_heads}
    if kind == "store":
        case["batch"] = _log_int(rng, 1, 128)
        case["count"] = rng.choice([1, _log_int(rng, 2, 8192)])
        case["count"] = max(1, min(case["count"], 250000 // (case["batch"] * (2 * kv_heads + case["q_heads"]))))
        return {**case, "past": _log_int(rng, 1, 8192), **_draw_turns(rng)}
    case |= {"window": _log_int(rng, 1, 8192), "sinks": rng.choice([0, 0, 1, 4, 64, 200]), "decodes": 0, "context": 0, "skew": False, "chunks": 0, "count": 0, "past": 0}
    form = rng.choice(["decode", "decode", "verify", "chunk", "mixed", "prompt"])
    if form in ("decode", "mixed"):
        case["decodes"] = _log_int(rng, 1, 96)
        case["skew"] = rng.random() < 0.5
        case["context"] = min(_log_int(rng, 64, 32768), max(64, 5000000 // (case["decodes"] * kv_heads)))
    if form != "decode":
        case["chunks"] = {"verify": _log_int(rng, 1, 32), "chunk": rng.choice([1, 1, 2, 4]), "mixed": rng.choice([1, 2, 3]), "prompt": rng.choice([1, 2, 5, 8])}[form]
        case["count"] = _log_int(rng, 2, 16) if form == "verify" else _log_int(rng, 17, 4096)
        case["past"] = 0 if form == "prompt" else _log_int(rng, 16, 32768)
        while case["q_heads"] * case["chunks"] * case["count"] * (min(case["past"], case["window"] + case["sinks"]) + case["count"]) > MOST_SCORES or \
                kv_heads * case["chunks"] * (case["past"] + case["count"]) > 720000:
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


def _axes(pairs, axes):
    """Axis of every pair: two axes take halves, three take turns until height and width are used up, the rest is time's."""
    if axes == 1:
        return [0] * pairs
    if axes == 2:
        return [i * 2 // pairs for i in range(pairs)]
    return [i % 3 if i < pairs // 8 * 6 else 0 for i in range(pairs)]


def _places(n, axes, at):
    """Positions [n][axes] of tokens whose places on the first axis are `at`: the other axes go over a picture's rows and columns."""
    side = max(2, math.isqrt(min(n, 1024)))
    return torch.stack([at.long()] + [torch.arange(n, device=DEV) // side ** (axes - 1 - a) % side for a in range(1, axes)], 1).int()


def _normed(x, w, case):
    """fp16 [tokens][heads][dim] -> 64 bits."""
    x = x.double()
    if case["norm"] == "none":
        return x
    if case["centred"]:
        x = x - x.mean(-1, keepdim=True)
    return x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * (w.double() + case["offset"])


def _rotate(x, positions, freq, axis, amp, layout):
    """64-bit [tokens][heads][dim], positions [tokens][axes] -> fp16, rotated.  In 64 bits: angles of far positions, and a value next to a
    code's border must not depend on the last bit of a sine."""
    half = freq.numel()
    angle = positions.double()[:, axis] * freq
    cos, sin = (angle.cos() * amp)[:, None], (angle.sin() * amp)[:, None]
    head, rest = x[..., :2 * half], x[..., 2 * half:]
    if layout == "half":
        a, b = head[..., :half], head[..., half:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((turned, rest), -1).float().half()


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

    def weights(self, case, heads, dim):
        """A norm's weights: around one, or around zero where one is added."""
        if case["norm"] == "none":
            return None
        w = torch.randn((heads, dim) if case["norm"] == "own" else (dim,), generator=self.g, device=DEV)
        return (0.2 * w + 1.0 - case["offset"]).half()

    def projected(self, *shape):
        """Heads as a projection leaves them: each with a size of its own, a little off centre."""
        x = torch.randn(shape, generator=self.g, device=DEV) + 0.1
        return (x * torch.randn(*shape[:2], 1, generator=self.g, device=DEV).exp()).half()


def _between(lo, hi, n):
    """n whole numbers from hi down to lo, evenly."""
    return [hi - (hi - lo) * i // max(n - 1, 1) for i in range(n)]


def _sequences(c):
    """(new tokens, cached tokens) of every sequence of a case: sizes go by the case, their order and all values by the seed."""
    if c["kind"] == "store":
        n, counts, past = c["batch"], _between((c["count"] + 1) // 2, c["count"], c["batch"]), _between(0, c["past"], c["batch"])
    elif c["kind"] == "pages":
        # rows without new tokens, decoding ones, and every eighth a prompt or its chunk
        n, idle = c["batch"], int(c["batch"] * c["idle"])
        counts = [0 if i < idle else c["count"] - c["count"] * (i % 5) // 9 if i % 8 == 7 else 1 for i in range(n)]
        past = _between(0, c["past"], n)
    else:
        # verification drafts as many tokens for every sequence; chunks and prompts are of different lengths
        n, lo = c["chunks"], c["count"] if c["count"] <= 16 else (c["count"] + 1) // 2
        counts, past = _between(lo, c["count"], n), _between((c["past"] + 1) // 2, c["past"], n)
    together = [(counts[i], past[i * 7 % n if n % 7 else i]) for i in range(n)]
    if c["kind"] == "window" and c["decodes"]:
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
    if c["kind"] in ("heads", "store"):
        f, state["amp"] = _frequencies(c["rot"], c["scaling"])
        state["freq"] = torch.tensor(f, dtype=torch.float64, device=DEV)
        state["axis"] = torch.tensor(_axes(c["rot"] // 2, c["axes"]), device=DEV)
        dim, k_heads = (c["dim"], c["k_heads"]) if c["kind"] == "heads" else (HEAD, c["kv_heads"])
        state["q_weight"], state["k_weight"] = r.weights(c, c["q_heads"], dim), r.weights(c, k_heads, dim)
    if own:                                              # the handles that a program makes once
        import paper_2508_15601_amd as tm
        if c["kind"] in ("heads", "store"):
            kind = {"none": tm.TM_ROPE_PLAIN, "linear": tm.TM_ROPE_LINEAR, "base": tm.TM_ROPE_BASE, "wavelength": tm.TM_ROPE_WAVELENGTH, "ramp": tm.TM_ROPE_RAMP}
            state["rope"] = tm.tm_rope_create(c["rot"], layout=tm.TM_ROPE_HALF if c["layout"] == "half" else tm.TM_ROPE_INTERLEAVED,
                                              base=BASE[c["scaling"]], scaling=kind[c["scaling"]], **SCALING[c["scaling"]],
                                              axis=_axes(c["rot"] // 2, c["axes"]) if c["axes"] > 1 else None)
            for x in "qk":
                w = state[x + "_weight"]
                state[x + "_norm"] = None if w is None else tm.HeadNorm(w, eps=EPS, offset=c["offset"], centred=c["centred"])
        if c["kind"] in ("store", "window"):
            state["cache"] = tm.tm_paged_create(*state["pool"])
            state["batch"] = tm.PagedBatch(state["table"], state["offsets"], state["positions"], max_count=max(state["counts"]),
                                           max_len=max(n + p for n, p in zip(state["counts"], state["past"])))
        if c["kind"] == "pages":
            # a pool of one KV head and 4-bit codes: its contents are not touched
            state["cache"] = tm.tm_paged_create(*tm.tm_paged_pool(state["pages"], 1, c["page"], bits=4))
            state["batch"] = tm.PagedBatch(state["table"], state["offsets"], state["positions"])
    return state


def run(state):
    return globals()["_own_" + state["case"]["kind"] if own else "_plain_" + state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------------------ heads

def _prepare_heads(c, r):
    n = c["tokens"]
    qk = r.projected(n, c["q_heads"] + c["k_heads"], c["dim"])           # what the fused projection left
    q, k = qk.split((c["q_heads"], c["k_heads"]), 1)
    at = torch.randint(0, c["far"], (n,), generator=r.g, device=DEV)
    return {"Q": q, "K": k, "Q_out": torch.empty_like(q, memory_format=torch.contiguous_format), "K_out": torch.empty_like(k, memory_format=torch.contiguous_format),
            "positions": at.int() if c["axes"] == 1 else _places(n, c["axes"], at)}


def _plain_heads(s):
    c = s["case"]
    at = s["positions"].view(c["tokens"], c["axes"])
    return [_rotate(_normed(x, w, c), at, s["freq"], s["axis"], s["amp"], c["layout"]) for x, w in ((s["Q"], s["q_weight"]), (s["K"], s["k_weight"]))]


def _own_heads(s):
    import paper_2508_15601_amd as tm
    tm.tm_heads_apply(rope=s["rope"], positions=s["positions"], Q=s["Q"], Q_out=s["Q_out"], q_norm=s["q_norm"], K=s["K"], K_out=s["K_out"], k_norm=s["k_norm"])
    return [s["Q_out"], s["K_out"]]


# ------------------------------------------------------------------------------------------------------------ store

def _prepare_store(c, r):
    Hq, Hk = c["q_heads"], c["kv_heads"]
    s = _batch(r, c)
    n = sum(s["counts"])
    q, k, v = r.projected(n, Hq + 2 * Hk, HEAD).split((Hq, Hk, Hk), 1)   # keys and values lie behind the queries
    new = lambda heads: torch.empty(n, heads, HEAD, dtype=torch.float16, device=DEV)  # noqa: E731
    return {**s, "pool": r.pool(s["pages"], Hk, c["page"], c["bits"], filled=False), "Q": q, "K": k, "V": v, "Q_out": new(Hq), "K_back": new(Hk), "V_back": new(Hk),
            "places": None if c["axes"] == 1 else _places(n, c["axes"], s["at"])}


def _plain_store(s):
    c = s["case"]
    at = s["at"][:, None] if s["places"] is None else s["places"]
    q, k = (_rotate(_normed(x, w, c), at, s["freq"], s["axis"], s["amp"], c["layout"]) for x, w in ((s["Q"], s["q_weight"]), (s["K"], s["k_weight"])))
    page, slot = _slots(s, c["page"])
    _store(s["pool"], page, slot, k, s["V"])
    k, v = _load(s["pool"], page, slot)
    return q, k.half(), v.half()


def _own_store(s):
    import paper_2508_15601_amd as tm
    tm.tm_paged_append(s["cache"], s["batch"], s["K"], s["V"], rope=s["rope"], Q=s["Q"], Q_out=s["Q_out"], q_norm=s["q_norm"], k_norm=s["k_norm"], positions=s["places"])
    tm.tm_paged_read(s["cache"], s["batch"], s["K_back"], s["V_back"])
    return s["Q_out"], s["K_back"], s["V_back"]


# ------------------------------------------------------------------------------------------------------------ pages

def _new_pages(c):
    """Pages that the sequences' new tokens begin."""
    return sum(-(-(n + p) // c["page"]) - -(-p // c["page"]) for n, p in _sequences(c))


def _prepare_pages(c, r):
    counts, past = map(list, zip(*r.shuffled(_sequences(c))))
    table, pages = r.table([p for p in past], c["page"]) if any(past) else (None, 0)
    wide = max(-(-(n + p) // c["page"]) for n, p in zip(counts, past)) + 2
    rows = torch.full((c["batch"], wide), -1, dtype=torch.int32, device=DEV)
    if table is not None:
        rows[:, :table.shape[1]] = table
    new = _new_pages(c)
    free = pages + torch.randperm(new + 5, generator=r.h)                # the pool has these besides the table's
    ints = lambda *n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
    return {"table": rows, "pages": pages + new + 5, "free": free.int().to(DEV),
            "available": torch.tensor([new * 3 // 4 if c["scarce"] else new + 5], dtype=torch.int32, device=DEV), "left": ints(1),
            "lens": torch.tensor(past, dtype=torch.int32, device=DEV), "counts": torch.tensor(counts, dtype=torch.int32, device=DEV), "lens_out": ints(c["batch"]),
            "offsets": ints(c["batch"] + 1), "positions": ints(c["batch"]), "short": ints(c["batch"]),
            "slots": torch.zeros(sum(counts), dtype=torch.int64, device=DEV)}


def _plain_pages(s):
    page, lens, counts = s["case"]["page"], s["lens"].long(), s["counts"].long()
    tokens, wide = s["slots"].numel(), s["table"].shape[1]
    ends = counts.cumsum(0)
    have = (lens + page - 1) // page
    need = (lens + counts + page - 1) // page - have
    taken = need.cumsum(0)
    short = (need > 0) & (taken > s["available"])
    served = ~short
    row = torch.searchsorted(ends, torch.arange(tokens, device=DEV), right=True)
    at = torch.arange(tokens, device=DEV) - (ends - counts)[row] + lens[row]
    number = at // page
    fresh = (s["available"] - 1 - (taken - need)[row] - number + have[row]).clamp(0, s["free"].numel() - 1)      # (of an old page: anything)
    entry = torch.where(number < have[row], s["table"][row, number], torch.where(short[row], -1, s["free"][fresh]))
    s["table"][row, number] = entry                      # every token of a page writes the same
    slots = torch.where(short[row], -1, entry.long() * page + at % page)
    left = s["available"] - (need * served).sum()
    return {"table": s["table"], "offsets": torch.cat((ends[:1] * 0, ends)).int(), "positions": lens.int(), "slots": slots, "short": short.int(),
            "lens": (lens + counts * served).int(), "left": left.int()}


def _own_pages(s):
    import paper_2508_15601_amd as tm
    tm.tm_paged_assign(s["cache"], tm.PageList(s["free"], s["available"]), s["batch"], s["lens"], s["counts"], slots=s["slots"], short=s["short"],
                       lens_out=s["lens_out"], left=s["left"])
    return {"table": s["table"], "offsets": s["offsets"], "positions": s["positions"], "slots": s["slots"], "short": s["short"], "lens": s["lens_out"], "left": s["left"]}


# ----------------------------------------------------------------------------------------------------------- window

def _prepare_window(c, r):
    s = _batch(r, c)
    q = r.normal(sum(s["counts"]), c["q_heads"], HEAD)
    return {**s, "pool": r.pool(s["pages"], c["kv_heads"], c["page"], c["bits"]), "Q": q, "O": torch.empty_like(q)}


def _plain_window(s):
    """Sequences with as many new tokens go together; of a context only the tokens are taken that a row sees: first ones, and those from the
    first row's window on."""
    c, out = s["case"], torch.empty_like(s["O"])
    Hk, G = c["kv_heads"], c["q_heads"] // c["kv_heads"]
    for n in sorted(set(s["counts"])):
        same = [b for b, m in enumerate(s["counts"]) if m == n]
        past = s["positions"][same].long()
        longest = max(s["past"][b] for b in same) + n
        lo = (past - c["window"] + 1).clamp_min(0)[:, None]                              # of a sequence's first row
        near = lo + torch.arange(min(longest, c["window"] - 1 + n), device=DEV)
        first = torch.arange(min(longest, c["sinks"]), device=DEV).expand(len(same), -1)
        t = torch.cat((first, near), 1)                                                  # [sequences][tokens]
        once = torch.cat((first < lo, near >= 0), 1)                                     # a first token inside the window is counted there
        longest = t.shape[1]
        page = s["table"][same].gather(1, (t // c["page"]).clamp_max(s["table"].shape[1] - 1)).clamp_min(0).long()      # behind a sequence: masked
        k, v = _load(s["pool"], page.flatten(), (t % c["page"]).flatten())
        k, v = (x.view(len(same), longest, Hk, HEAD).transpose(1, 2).contiguous() for x in (k, v))
        rows = s["offsets"][same].long()[:, None] + torch.arange(n, device=DEV)
        q = s["Q"][rows].float().view(len(same), n, Hk, G, HEAD).permute(0, 2, 1, 3, 4).reshape(len(same), Hk, n * G, HEAD)
        x = torch.matmul(q, k.transpose(2, 3)).mul_(ROOT).view(len(same), Hk, n, G, longest)
        p = (past[:, None] + torch.arange(n, device=DEV))[:, :, None]                    # [sequences][n][1]
        seen = once[:, None] & (t[:, None] <= p) & ((t[:, None] > p - c["window"]) | (t[:, None] < c["sinks"]))
        x = x.masked_fill_(~seen[:, None, :, None], -math.inf)
        x = (x - x.amax(-1, keepdim=True)).exp_()
        x = x.div_(x.sum(-1, keepdim=True)).view(len(same), Hk, n * G, longest)
        o = torch.matmul(x, v).view(len(same), Hk, n, G, HEAD).permute(0, 2, 1, 3, 4)
        out[rows] = o.reshape(len(same), n, c["q_heads"], HEAD).half()
    return out


def _own_window(s):
    import paper_2508_15601_amd as tm
    c = s["case"]
    return tm.tm_paged_attn(s["Q"], s["cache"], s["batch"], s["O"], ROOT, window=c["window"], sinks=c["sinks"])


# ----------------------------------------------------------------------------------------------------- work, exact

def _token_bytes(bits):
    """Codes and pairs of one token and KV head, key and value."""
    return 2 * HEAD * bits // 8 + 8


def _seen(past, n, window, sinks):
    """(pairs of a row and a token it sees, tokens that any row sees) of a sequence."""
    rows = range(past, past + n)
    pairs = sum(min(p + 1, window) + min(sinks, max(p + 1 - window, 0)) for p in rows)
    lo = max(past - window + 1, 0)
    return pairs, past + n - lo + min(sinks, lo)


def work(case):
    c, kind = case, case["kind"]
    if kind == "heads":
        heads = c["q_heads"] + c["k_heads"]
        weights = {"none": 0, "shared": 4 * c["dim"], "own": 2 * heads * c["dim"]}[c["norm"]]
        return {"bytes": c["tokens"] * (4 * heads * c["dim"] + 4 * c["axes"]) + weights,
                "flops": float(c["tokens"]) * heads * (3 * c["rot"] + (0 if c["norm"] == "none" else 4 * c["dim"]))}
    seqs = _sequences(c)
    n = sum(m for m, _ in seqs)
    if kind == "store":
        moved = c["kv_heads"] * (2 * _token_bytes(c["bits"]) + 8 * HEAD) + 4 * c["q_heads"] * HEAD
        norms = 0 if c["norm"] == "none" else 4
        return {"bytes": n * moved, "flops": n * HEAD * ((13.0 + norms) * c["kv_heads"] + (3.0 + norms) * c["q_heads"])}
    if kind == "pages":
        return {"bytes": c["batch"] * 24 + 8 * n + 8 * _new_pages(c), "flops": 8.0 * n + 8.0 * c["batch"]}
    seen = [_seen(past, m, c["window"], c["sinks"]) for m, past in seqs]
    return {"bytes": sum(t for _, t in seen) * c["kv_heads"] * _token_bytes(c["bits"]) + 4 * n * c["q_heads"] * HEAD,
            "flops": 4.0 * HEAD * c["q_heads"] * sum(p for p, _ in seen)}


def _stored64(x, bits):
    """What a quantised cache holds for the vectors x (64 bits): scale to fp16, codes to the nearest."""
    top = 2 ** bits - 1
    lo, hi = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
    scale = ((hi - lo) / top).float().half().double()
    scale[scale == 0] = 1.0
    zero = torch.clamp(torch.round(-lo / scale), 0, top)
    return (torch.clamp(torch.round(x / scale) + zero, 0, top) - zero) * scale


def _normed64(x, w, c):
    x = x.to(torch.float64)
    if c["norm"] == "none":
        return x
    dim = x.shape[-1]
    mean = x.sum(-1, keepdim=True) / dim if c["centred"] else torch.zeros_like(x[..., :1])
    power = torch.pow(x - mean, 2).sum(-1, keepdim=True) / dim
    return (x - mean) * torch.pow(power + EPS, -0.5) * (c["offset"] + w.to(torch.float64))


def _turned64(x, at, c):
    """Rotation as a product of complex numbers; x [n][heads][dim], at [n][axes]."""
    f, amp = _frequencies(c["rot"], c["scaling"])
    angle = torch.stack([at[:, a].double() * w for w, a in zip(f, _axes(c["rot"] // 2, c["axes"]))], 1)
    turn = torch.polar(torch.full((1, 1), amp, dtype=torch.float64, device=DEV), angle)[:, None]
    y = x.clone()
    first, second = (slice(0, c["rot"] // 2), slice(c["rot"] // 2, c["rot"])) if c["layout"] == "half" else (slice(0, c["rot"], 2), slice(1, c["rot"], 2))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _pages_by_hand(s):
    """Row after row."""
    page, free = s["case"]["page"], s["free"].tolist()[:int(s["available"])]
    table, lens, counts = s["table"].tolist(), s["lens"].tolist(), s["counts"].tolist()
    offsets, slots, short, out, asked = [0], [], [], [], 0
    available = len(free)
    for b, (n, new) in enumerate(zip(lens, counts)):
        need = len(range(-(-n // page), -(-(n + new) // page)))
        asked += need
        denied = need > 0 and asked > available
        for j in range(need):
            table[b][-(-n // page) + j] = -1 if denied else free.pop()
        slots += [-1 if denied else table[b][t // page] * page + t % page for t in range(n, n + new)]
        offsets.append(offsets[-1] + new)
        short.append(int(denied))
        out.append(n if denied else n + new)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    return {"table": ints(table), "offsets": ints(offsets), "positions": ints(lens), "slots": torch.tensor(slots, dtype=torch.int64, device=DEV), "short": ints(short),
            "lens": ints(out), "left": ints([len(free)])}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "heads":
        at = s["positions"].view(c["tokens"], c["axes"])
        return [_turned64(_normed64(x, w, c), at, c) for x, w in ((s["Q"], s["q_weight"]), (s["K"], s["k_weight"]))]
    if c["kind"] == "store":
        at = s["at"][:, None] if s["places"] is None else s["places"]
        q, k = (_turned64(_normed64(x, w, c), at, c) for x, w in ((s["Q"], s["q_weight"]), (s["K"], s["k_weight"])))
        return q, _stored64(k.float().half().double(), c["bits"]), _stored64(s["V"].double(), c["bits"])        # a key is stored from its fp16 value
    if c["kind"] == "pages":
        return _pages_by_hand(s)
    out, row = [], 0
    for b, n in enumerate(s["counts"]):                  # sequence by sequence, long chunks one head at a time
        past, G = s["past"][b], c["q_heads"] // c["kv_heads"]
        t = torch.arange(past + n, device=DEV)
        t = t[(t < c["sinks"]) | (t > past - c["window"])]
        k, v = _codes64(s["pool"], s["table"][b, t // c["page"]].long(), t % c["page"])
        p = torch.arange(past, past + n, device=DEV)[:, None]
        mask = (t > p) | ((t >= c["sinks"]) & (p - t >= c["window"]))
        q, heads = s["Q"][row:row + n].double().transpose(0, 1), []
        for h in range(c["q_heads"]):
            logits = torch.where(mask, -math.inf, q[h] @ k[:, h // G].T.contiguous() / math.sqrt(HEAD))
            heads.append(torch.softmax(logits, -1) @ v[:, h // G].contiguous())
        out.append(torch.stack(heads).transpose(0, 1))
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
