"""The measured operators of the LLM task's side of the hand-off: queries and keys normed and rotated, the 4-bit cache
written and read back, and attention over it.

A state holds what a serving program has in hand before the call: the packed QKV rows of a layer, the rotary table, the
cache's pool of pages with its page table, slots and lengths.  Where ``own`` is false the operators run in their plain
form, elementary torch operations in fp32; where it is true, through the framework's calls.

A case is a plain dict.  ``op`` is

* "qk"     ``rows`` tokens of packed QKV; ``axes`` 1 or 3 position axes, ``sections`` "contiguous" or "interleaved",
           ``rotary`` values of a head that rotate, ``norm`` whether queries and keys are normed, ``dtype``;
* "write"  ``rows`` tokens quantised into the pool and read back as the values they are held as;
* "read"   ``rows`` tokens of a filled pool read as values;
* "attend" ``batch`` sequences of at most ``queries`` new tokens and ``longest`` keys (``ragged``: lengths from 1 % of
           that; ``idle``: that many padding sequences without keys), ``causal``; ``lens`` draws the lengths.

Pages are ``page`` tokens, in no order.  A page holds, per key/value head, K codes, V codes, K scales and V scales; a group of
32 values has one power of two (a byte, exponent + 127) and 32 codes of 4 bits (sign, and an index into 0 .5 1 1.5 2 3 4 6).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
GROUP = 32                  # values that share a scale
THETA, EPS = 1e6, 1e-6
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ---------------------------------------------------------------------------------------------------
def _qk(rows, heads, kv_heads, dim, rotary, axes=3, sections="contiguous", norm=True, dtype="bf16"):
    return {"op": "qk", "rows": rows, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rotary": rotary, "axes": axes,
            "sections": sections, "norm": norm, "dtype": dtype}


def _rows(op, rows, kv_heads, dim, page, dtype="bf16"):
    return {"op": op, "rows": rows, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype}


def _attend(batch, queries, longest, heads, kv_heads, dim, page, ragged=False, idle=0, causal=True, lens=0):
    return {"op": "attend", "batch": batch, "queries": queries, "longest": longest, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "page": page, "ragged": ragged, "idle": idle, "causal": causal, "lens": lens}


def listed():
    return [
        # one generated token of a layer of 3584 (the width of the 7B-style towers' embeddings): latency alone
        {"name": "qk_token", **_qk(1, 28, 4, 128, 128)},
        # an image prompt of the small fp32 layer, an odd number of rows, axes interleaved over the frequencies
        {"name": "qk_1125_f32", **_qk(1125, 8, 2, 64, 64, sections="interleaved", dtype="f32")},
        # two clips' sequences, prefilled at once
        {"name": "qk_video_16384", **_qk(16384, 28, 4, 128, 128)},
        # the new tokens of a decode batch, one row in each sequence's last page
        {"name": "write_48", **_rows("write", 48, 8, 128, 64)},
        # a packed prompt batch of sixteen thousand tokens
        {"name": "write_16384", **_rows("write", 16384, 8, 128, 128)},
        # a prompt's cached prefix handed to another layer's code in fp32, heads of 64
        {"name": "read_5001_f32", **_rows("read", 5001, 2, 64, 32, dtype="f32")},
        # a long shared prefix read as bf16 rows
        {"name": "read_65536", **_rows("read", 65536, 4, 128, 64)},
        # one sequence, one token: the smallest step of a chat
        {"name": "attend_token_2048", **_attend(1, 1, 2048, 28, 4, 128, 64)},
        # one token against a long document or film
        {"name": "attend_long_131072", **_attend(1, 1, 131072, 28, 4, 128, 128)},
        # a decode batch of ragged sequences, padded with idle rows as a recorded graph pads it
        {"name": "attend_batch_64", **_attend(64, 1, 16384, 28, 4, 128, 64, ragged=True, idle=3, lens=1)},
        # drafted tokens of a few sequences checked at once, odd lengths
        {"name": "attend_draft_6x5", **_attend(6, 5, 4097, 32, 8, 128, 32, ragged=True, lens=2)},
        # a chunk of a prompt behind fourteen thousand cached tokens
        {"name": "attend_chunk_2048", **_attend(1, 2048, 16384, 28, 4, 128, 128)},
    ]


_HEADS = ((28, 4, 128), (32, 8, 128), (16, 16, 128), (8, 1, 128), (8, 2, 64), (20, 20, 64), (32, 4, 64))


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["qk", "qk", "write", "write", "read", "attend", "attend", "attend", "attend", "attend"])
    heads, kv_heads, dim = rng.choice(_HEADS)
    page = rng.choice([32, 32, 64, 64, 96, 128, 256])
    if op == "qk":
        most = 16384 * 32 * 128 // ((heads + kv_heads) * dim)
        axes = rng.choice([1, 3, 3])
        return _qk(min(_log_int(rng, 1, 16384), most), heads, kv_heads, dim, rng.choice([dim, dim, dim // 2]), axes,
                   rng.choice(["contiguous", "interleaved"]) if axes == 3 else "contiguous", rng.random() < 0.7,
                   "bf16" if rng.random() < 0.7 or heads * dim > 2048 else "f32")
    if op in ("write", "read"):
        most = (16384 if op == "write" else 32768) * 8 * 128 // (kv_heads * dim)
        return _rows(op, min(_log_int(rng, 1, 16384 if op == "write" else 65536), most // 2), kv_heads, dim, page, rng.choice(["bf16", "bf16", "f32"]))
    kind, lens, causal = rng.choice(["decode", "decode", "draft", "long", "chunk", "chunk"]), rng.randrange(1 << 20), rng.random() < 0.85
    room = 64 * 16384 * 4 * 128 // (2 * kv_heads * dim)        # padded keys of a batch
    if kind == "long":
        return _attend(rng.choice([1, 1, 2]), 1, min(_log_int(rng, 16384, 131072), room), heads, kv_heads, dim, page, causal=causal, lens=lens)
    if kind == "chunk":
        queries = _log_int(rng, 16, 2048)
        batch = rng.randint(1, max(1, min(8, 2048 // queries)))
        longest = queries + _log_int(rng, 1, 8192)
        return _attend(batch, queries, longest, heads, kv_heads, dim, page, ragged=batch > 1, causal=causal, lens=lens)
    batch, queries = _log_int(rng, 1, 64), 1 if kind == "decode" else rng.randint(2, 8)
    longest = max(queries, min(_log_int(rng, 16, 16384), room // batch))
    return _attend(batch, queries, longest, heads, kv_heads, dim, page, ragged=rng.random() < 0.7, idle=batch // 16 * rng.randint(0, 2), causal=causal, lens=lens)


def _lengths(case):
    """[(queries, keys), ...] of the sequences: the first is the longest; an idle one has a row of queries and no keys."""
    r, q, n = random.Random(case["lens"]), case["queries"], case["longest"]
    got = [(q, n)]
    for b in range(1, case["batch"]):
        idle = b >= case["batch"] - case["idle"]
        keys = max(1, _log_int(r, max(1, n // 100), n)) if case["ragged"] else n
        got.append((1, 0) if idle else (min(keys, r.randint(1, q) if case["ragged"] and q > 8 else q), keys))
    return got


# ---- the cache's layout ----------------------------------------------------------------------------------------
def _block(page, dim):
    """Bytes of a page's part of one head."""
    return page * (dim + 2 * (dim // GROUP))


def _places(slots, heads, dim, page):
    """Byte addresses in the pool of the K codes, V codes [rows, heads, dim / 2], K scales and V scales [rows, heads, dim / 32] of
    slots (page number * page + token within it)."""
    ng, wide = dim // GROUP, dim // 16
    tok = (slots % page)[:, None, None]
    base = ((slots // page)[:, None] * heads + torch.arange(heads, device=slots.device)) * _block(page, dim)
    base = base[:, :, None]
    d = torch.arange(0, dim, 2, device=slots.device)
    g = torch.arange(ng, device=slots.device)
    k = tok * (dim // 2) + ((d % 32 // 8) * ng + d // 32) * 4 + d % 8 // 2
    v = page * dim // 2 + tok // 4 * (2 * dim) + d // wide * (4 * dim // 32) + tok % 4 * (dim // 32) + d % wide // 2
    ks = page * dim + tok * ng + g
    vs = page * (dim + ng) + tok // 8 * (8 * ng) + g * 8 + tok % 8
    return base + k, base + v, base + ks, base + vs


def _quantise(x):
    """[rows, heads, dim] fp32 -> (bytes of two codes [rows, heads, dim / 2], scale bytes [rows, heads, dim / 32])."""
    x = torch.nan_to_num(x, nan=0.0, posinf=torch.finfo(torch.float32).max, neginf=torch.finfo(torch.float32).min)
    x = x.view(*x.shape[:-1], -1, GROUP)
    byte = ((x.abs().amax(-1).view(torch.int32) + 0x200000 >> 23) - 2).clamp(2, 252)
    y = x * (254 - byte << 23).view(torch.float32)[..., None]
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6.0)
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.int32) + 8 * (y < 0)
    code = code.flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), byte.to(torch.uint8)


def _values(codes, scales):
    """The reverse of _quantise, fp32."""
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=codes.device)
    y = level[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    power = (scales.int() << 23).view(torch.float32)
    return (y.view(*scales.shape, GROUP) * power[..., None]).flatten(-2)


# ---- states ----------------------------------------------------------------------------------------------------
class _State:
    pass


def _sections(case):
    half, axes = case["rotary"] // 2, case["axes"]
    if axes == 1:
        return (half,)
    if case["sections"] == "interleaved":          # a third each, the rest to time
        return (half - 2 * (half // 3), half // 3, half // 3)
    return (half // 4, half // 4 + half // 8, half - 2 * (half // 4) - half // 8)


def _axis_of(case):
    """Axis of each rotary pair."""
    sec, half = _sections(case), case["rotary"] // 2
    if case["sections"] == "interleaved":
        return [j % 3 if j % 3 and j < 3 * sec[j % 3] else 0 for j in range(half)]
    return [a for a, n in enumerate(sec) for _ in range(n)]


def _prepare_qk(s, case, gen):
    T, H, K, D = case["rows"], case["heads"], case["kv_heads"], case["dim"]
    dtype = TYPES[case["dtype"]]
    s.qkv = torch.randn(T, (H + 2 * K) * D, generator=gen, device=DEV).to(dtype)
    s.q = s.qkv[:, :H * D].view(T, H, D)
    s.k = s.qkv[:, H * D:(H + K) * D].view(T, K, D)
    s.q_gain = s.k_gain = None
    if case["norm"]:
        s.q_gain, s.k_gain = (1 + 0.1 * torch.randn(D, generator=gen, device=DEV) for _ in range(2))
    # text, then frames of a grid 24 wide: time, height and width advance as in a film
    t = torch.arange(T, device=DEV) + int(torch.randint(0, 1000, (1,), generator=gen, device=DEV))
    s.positions = t[:, None] if case["axes"] == 1 else torch.stack((t // 384, t // 24 % 16, t % 24), -1) + t[:1, None] // 2
    s.positions = s.positions.int().contiguous()
    n = int(s.positions.max()) + 1
    half = case["rotary"] // 2
    angle = torch.arange(n, device=DEV, dtype=torch.float64)[:, None] * THETA ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    s.cos_sin = torch.stack((angle.cos(), angle.sin()), -1).float()
    s.sections, s.interleaved = _sections(case), case["sections"] == "interleaved"
    s.axis = torch.tensor(_axis_of(case), device=DEV)


def _keys(rows, heads, dim, gen):
    """Keys and values of a layer: keys with a few channels that stand out."""
    loud = 1 + 3 * (torch.rand(heads, dim, generator=gen, device=DEV) < 0.05)
    k = torch.randn(rows, heads, dim, generator=gen, device=DEV) * loud
    return k.bfloat16(), torch.randn(rows, heads, dim, generator=gen, device=DEV).bfloat16()


def _pool(pages, heads, dim, page, gen):
    """A pool as it is found: memory with anything in it."""
    return torch.randint(0, 256, (pages, heads * _block(page, dim)), generator=gen, device=DEV, dtype=torch.uint8)


def _fill(pool, slots, k, v, page):
    places = _places(slots, k.shape[1], k.shape[2], page)
    flat = pool.view(-1)
    (kc, ks), (vc, vs) = _quantise(k.float()), _quantise(v.float())
    flat[places[0]], flat[places[1]], flat[places[2]], flat[places[3]] = kc, vc, ks, vs


def _prepare_rows(s, case, gen):
    T, H, D, P = case["rows"], case["kv_heads"], case["dim"], case["page"]
    pages = -(-T // P) + 2 if T > 64 else T + 2
    s.pool = _pool(pages, H, D, P, gen)
    order = torch.randperm(pages, generator=gen, device=DEV)
    t = torch.arange(T, device=DEV)
    if T > 64:      # a prompt: page after page
        s.slots = order[t // P] * P + t % P
    else:           # one row in each sequence's own page
        s.slots = order[t] * P + torch.randint(0, P, (T,), generator=gen, device=DEV)
    k, v = _keys(T, H, D, gen)
    if case["op"] == "read":
        _fill(s.pool, s.slots, k, v, P)
        if T > 64:
            s.slots[T // 2] = -1        # a row that nothing is held of
    else:           # rows of the packed QKV of the layer, queries in front
        s.kv = torch.cat((torch.zeros_like(k), k, v), 1).to(TYPES[case["dtype"]])
        s.k, s.v = s.kv[:, H:2 * H], s.kv[:, 2 * H:]


def _prepare_attend(s, case, gen):
    H, K, D, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    lens = np.asarray(_lengths(case), np.int64)
    need = -(-lens[:, 1] // P)
    width, pages = max(1, int(need.max())), int(need.sum()) + 1
    order = torch.randperm(pages, generator=gen, device=DEV).int()
    s.table = torch.full((len(lens), width), -1, device=DEV, dtype=torch.int32)
    held = torch.arange(width, device=DEV)[None] < torch.from_numpy(need).to(DEV)[:, None]
    s.table[held] = order[:pages - 1]
    s.n_keys = torch.from_numpy(lens[:, 1]).to(DEV).int()
    s.cu = torch.from_numpy(np.concatenate([[0], np.cumsum(lens[:, 0])])).to(DEV).int()
    s.q = torch.randn(int(lens[:, 0].sum()), H, D, generator=gen, device=DEV).bfloat16()
    s.pool = _pool(pages, K, D, P, gen)
    t = torch.arange(width * P, device=DEV)
    slots = (s.table.long()[:, t // P] * P + t % P)[t[None] < s.n_keys[:, None]]
    for part in slots.split(1 << 17):
        _fill(s.pool, part, *_keys(len(part), K, D, gen), P)
    s.max_queries, s.max_keys = int(lens[:, 0].max()), int(lens[:, 1].max())


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    s = _State()
    s.case = case
    {"qk": _prepare_qk, "write": _prepare_rows, "read": _prepare_rows, "attend": _prepare_attend}[case["op"]](s, case, gen)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------
def _plain_norm_rope(s, x, gain):
    half = s.case["rotary"] // 2
    y = x.float()
    if gain is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS) * gain
    cs = s.cos_sin[s.positions[:, s.axis], torch.arange(half, device=DEV)]
    c, n = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = y[..., :half], y[..., half:2 * half]
    return torch.cat((a * c - b * n, b * c + a * n, y[..., 2 * half:]), -1).to(x.dtype)


def _plain_read(pool, slots, heads, dim, page):
    """Keys and values [rows, heads, dim] fp32; a negative slot reads as zeros."""
    places = _places(slots.clamp(min=0), heads, dim, page)
    flat, held = pool.view(-1), (slots >= 0)[:, None, None]
    k = torch.where(held, _values(flat[places[0]], flat[places[2]]), 0.0)
    return k, torch.where(held, _values(flat[places[1]], flat[places[3]]), 0.0)


def _plain_attend(s):
    H, K, D, P = (s.case[n] for n in ("heads", "kv_heads", "dim", "page"))
    B, N, Q = len(s.n_keys), s.max_keys, s.max_queries
    t, i = torch.arange(N, device=DEV), torch.arange(Q, device=DEV)
    slots = s.table.long()[:, t // P] * P + t % P
    held = t[None] < s.n_keys[:, None]
    k, v = _plain_read(s.pool, torch.where(held, slots, -1).view(-1), K, D, P)
    k, v = (x.view(B, N, K, D).transpose(1, 2).contiguous() for x in (k, v))
    nq = s.cu[1:] - s.cu[:-1]
    row = (s.cu[:-1, None] + i).clamp(max=len(s.q) - 1).long()
    q = s.q.float()[row].view(B, Q, K, H // K, D).permute(0, 2, 3, 1, 4).reshape(B, K, H // K * Q, D)
    score = (q @ k.transpose(2, 3).contiguous()) * D ** -0.5
    see = held[:, None]
    if s.case["causal"]:
        see = see & (t[None, None] <= (s.n_keys - nq)[:, None, None] + i[None, :, None])
    see = see.expand(B, Q, N)[:, None, None]
    score = score.view(B, K, H // K, Q, N).masked_fill(~see, -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
    p = (p / p.sum(-1, keepdim=True).clamp(min=1e-30)).view(B, K, H // K * Q, N)
    out = (p @ v).view(B, K, H // K, Q, D).permute(0, 3, 1, 2, 4).reshape(B, Q, H, D)
    return out[i[None] < nq[:, None]].to(s.q.dtype)


def run(state):
    s, case = state, state.case
    if own:
        from paper_2603_12118_amd import binding as B
        if case["op"] == "qk":
            q, k = B.cs_qk_norm_rope(s.q, s.k, s.cos_sin, s.positions, s.sections, q_gain=s.q_gain, k_gain=s.k_gain, eps=EPS,
                                     interleaved=s.interleaved)
            return {"q": q, "k": k}
        if case["op"] == "attend":
            return B.cs_attention_cache(s.q, s.pool, s.table, s.n_keys, s.cu, s.max_queries, s.max_keys, case["kv_heads"], case["page"],
                                        causal=case["causal"])
        if case["op"] == "write":
            B.cs_cache_write(s.pool, s.k, s.v, s.slots, case["page"])
        k, v = B.cs_cache_read(s.pool, s.slots, case["kv_heads"], case["dim"], case["page"], dtype=TYPES[case["dtype"]])
        return {"k": k, "v": v}
    if case["op"] == "qk":
        return {"q": _plain_norm_rope(s, s.q, s.q_gain), "k": _plain_norm_rope(s, s.k, s.k_gain)}
    if case["op"] == "attend":
        return _plain_attend(s)
    if case["op"] == "write":
        _fill(s.pool, s.slots, s.k, s.v, case["page"])
    k, v = _plain_read(s.pool, s.slots, case["kv_heads"], case["dim"], case["page"])
    return {"k": k.to(TYPES[case["dtype"]]), "v": v.to(TYPES[case["dtype"]])}


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    D, K = case["dim"], case["kv_heads"]
    held = 2 * K * (D // 2 + D // GROUP)            # bytes of a token in the cache
    if case["op"] == "attend":
        H, pairs = case["heads"], 0
        lens = _lengths(case)
        for q, n in lens:
            pairs += q * n if not case["causal"] else q * n - q * (q - 1) // 2 if q <= n else n * (n + 1) // 2
        rows = sum(q for q, _ in lens)
        return {"bytes": float(sum(n for _, n in lens) * held + 4 * rows * H * D), "flops": float(4 * D * H * pairs)}
    T, size = case["rows"], 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "qk":
        values = T * (case["heads"] + K) * D
        return {"bytes": float(2 * values * size + T * 4 * (case["rotary"] + case["axes"])), "flops": float(8 * values)}
    values = 2 * T * K * D
    if case["op"] == "write":                       # rows in, the cache written and read, values out
        return {"bytes": float(2 * values * size + 2 * T * held + 16 * T), "flops": float(4 * values)}
    return {"bytes": float(values * size + T * held + 8 * T), "flops": float(values)}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------
def _two_to(e):
    """2^e in fp64, e a tensor of whole numbers."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _exact_held(x):
    """The values that [..., dim] is held as: per 32 of them, the nearest level at the group's power of two."""
    x = x.double()
    x = torch.where(x.isnan(), 0.0, x).reshape(*x.shape[:-1], -1, 32)
    top = x.abs().amax(-1, keepdim=True)
    mantissa, exponent = torch.frexp(top)           # top = mantissa 2^exponent, 1/2 <= mantissa < 1
    e = (exponent - 3 + (mantissa >= 0.875)).clamp(-125, 125)
    e = torch.where(top == 0, -125, e)
    y = x.abs() * _two_to(-e)
    index = torch.zeros_like(y, dtype=torch.long)
    for n, (lo, hi) in enumerate(zip(LEVELS[:-1], LEVELS[1:])):
        mid = (lo + hi) / 2
        index += (y > mid) | ((y == mid) & (n % 2 == 1))        # a tie goes to the even code
    level = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)[index]
    return (level * _two_to(e) * x.sign()).flatten(-2)


def _exact_page(block, dim, page):
    """One head's bytes of pages [n, block] -> keys, values [n * page, dim]."""
    n, ng = len(block), dim // 32
    def part(at, size):
        return block[:, at:at + size]
    def value(codes, power):
        level = torch.tensor(LEVELS, dtype=torch.float64, device=block.device)
        two = torch.stack((codes % 16, codes // 16), -1).flatten(-2).long()
        y = torch.where(two >= 8, -level[two % 8], level[two % 8])
        return (y.reshape(n * page, ng, 32) * _two_to(power.reshape(n * page, ng, 1).int() - 127)).view(n * page, dim)
    k = part(0, page * dim // 2).reshape(n, page, 4, ng, 4).permute(0, 1, 3, 2, 4).reshape(n, page, dim // 2)
    v = part(page * dim // 2, page * dim // 2).reshape(n, page // 4, 16, 4, dim // 32).permute(0, 1, 3, 2, 4).reshape(n, page, dim // 2)
    ks = part(page * dim, page * ng).reshape(n, page, ng)
    vs = part(page * (dim + ng), page * ng).reshape(n, page // 8, ng, 8).permute(0, 1, 3, 2).reshape(n, page, ng)
    return value(k, ks), value(v, vs)


def _exact_attend(s):
    H, K, D, P = (s.case[n] for n in ("heads", "kv_heads", "dim", "page"))
    out = torch.zeros(len(s.q), H, D, dtype=torch.float64, device=DEV)
    at, keys = s.cu.tolist(), s.n_keys.tolist()
    blocks = s.pool.view(len(s.pool), K, -1)
    for b, n in enumerate(keys):
        if not n:
            continue
        used = s.table[b, :-(-n // P)].long()
        last = torch.arange(n, device=DEV)
        place = n - (at[b + 1] - at[b]) + torch.arange(at[b + 1] - at[b], device=DEV)
        for h in range(K):
            k, v = (x[:n] for x in _exact_page(blocks[used, h], D, P))
            for g in range(h * (H // K), (h + 1) * (H // K)):
                w = s.q[at[b]:at[b + 1], g].double() @ k.T / math.sqrt(D)
                if s.case["causal"]:
                    w = torch.where(last[None] <= place[:, None], w, -math.inf)
                out[at[b]:at[b + 1], g] = torch.nan_to_num(torch.softmax(w, -1), nan=0.0) @ v
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(s)
    if case["op"] == "write":
        return {"k": _exact_held(s.k), "v": _exact_held(s.v)}
    if case["op"] == "read":
        P, D, got = case["page"], case["dim"], {"k": [], "v": []}
        for h in range(case["kv_heads"]):
            k, v = _exact_page(s.pool.view(len(s.pool), case["kv_heads"], -1)[:, h], D, P)
            for name, x in (("k", k), ("v", v)):
                x = x[s.slots.clamp(min=0)]
                x[s.slots < 0] = 0.0
                got[name].append(x)
        return {n: torch.stack(x, 1) for n, x in got.items()}
    out = {}
    for name, x, gain in (("q", s.q, s.q_gain), ("k", s.k, s.k_gain)):
        y = x.double()
        if gain is not None:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * gain.double()
        z, half = y.clone(), case["rotary"] // 2
        for j, a in enumerate(_axis_of(case)):
            c, n = (s.cos_sin.double()[s.positions[:, a].long(), j, i][:, None] for i in (0, 1))
            z[..., j] = y[..., j] * c - y[..., j + half] * n
            z[..., j + half] = y[..., j + half] * c + y[..., j] * n
        out[name] = z
    return out
