"""CPU oracle of the LLM task's attention calls: rotation and norm, the 4-bit cache, attention over it.

Written from the definitions in include/cornenc.h, in numpy fp64, row by row and head by head; test infrastructure only.
"""
from __future__ import annotations

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
F32_MAX = float(np.finfo(np.float32).max)


# ---- rotation and norm
def axis_of_pairs(sections, interleaved: bool):
    """The position axis each rotary pair follows."""
    half = int(sum(sections))
    if interleaved:
        return np.array([j % 3 if j % 3 and j < 3 * sections[j % 3] else 0 for j in range(half)])
    return np.repeat(np.arange(len(sections)), sections)


def norm_rope(x, cos_sin, positions, sections, gain=None, eps=1e-6, interleaved=False):
    """x [T, heads, D] -> [T, heads, D] fp64; cos_sin [n, half, 2], positions [T, axes]."""
    y = np.asarray(x, np.float64)
    if gain is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(gain, np.float64)
    axis, half = axis_of_pairs(sections, interleaved), int(sum(sections))
    cs = np.asarray(cos_sin, np.float64)[np.asarray(positions)[:, axis], np.arange(half)]       # [T, half, 2]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    out = y.copy()
    out[..., :half] = y[..., :half] * c - y[..., half:2 * half] * s
    out[..., half:2 * half] = y[..., half:2 * half] * c + y[..., :half] * s
    return out


# ---- the cache
def quantise(x):
    """x [..., D] -> (codes [..., D] 0..15, exponent bytes [..., D/32]); the nearest level, ties to the even code."""
    x = np.asarray(x, np.float64)
    x = np.clip(np.where(np.isnan(x), 0.0, x), -F32_MAX, F32_MAX)
    g = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(g).max(-1)
    mantissa, exponent = np.frexp(top)                     # top = mantissa 2^exponent, mantissa in [1/2, 1)
    e = np.clip(exponent - 1 - 2 + (2 * mantissa >= 1.75), -125, 125)
    e = np.where(top == 0, -125, e)
    y = np.ldexp(np.abs(g), -e[..., None])
    dist = np.abs(y[..., None] - LEVELS)
    best = dist.min(-1, keepdims=True)
    tied = dist == best                                    # one level, or two neighbours
    even = tied & (np.arange(8) % 2 == 0)
    code = np.where(tied.sum(-1) > 1, even.argmax(-1), tied.argmax(-1))
    code = code + 8 * np.signbit(g)
    return code.reshape(x.shape).astype(np.uint8), (e + 127).astype(np.uint8)


def values(codes, scales):
    """The reverse of quantise, fp64 (exact)."""
    v = np.where(codes >= 8, -1.0, 1.0) * LEVELS[codes & 7]
    return np.ldexp(v.reshape(*scales.shape, 32), scales.astype(np.int64)[..., None] - 127).reshape(codes.shape)


def held(x):
    """The values x [..., D] is held as."""
    return values(*quantise(x))


def code_addresses(o: int, page_tokens: int, dim: int):
    """Of token o of a block: byte offsets of the K and V codes of dims (0, 1), (2, 3) ... and of the K and V scales of each group."""
    ng, d, g = dim // 32, np.arange(0, dim, 2), np.arange(dim // 32)
    k = o * dim // 2 + (d % 32 // 8 * ng + d // 32) * 4 + d % 8 // 2
    v = page_tokens * dim // 2 + o // 4 * 2 * dim + d // (dim // 16) * 4 * ng + o % 4 * ng + d % (dim // 16) // 2
    return k, v, page_tokens * dim + o * ng + g, page_tokens * (dim + ng) + o // 8 * 8 * ng + 8 * g + o % 8


def write(pool, k, v, slots, page_tokens: int):
    """A copy of pool [n_pages, page bytes] with the rows k, v [T, heads, D] written at their slots (a negative or too large one: skipped)."""
    T, heads, dim = k.shape
    out = pool.copy()
    block = page_tokens * (dim + 2 * (dim // 32))
    for t, slot in enumerate(slots):
        if not 0 <= slot < len(pool) * page_tokens:
            continue
        page, o = divmod(int(slot), page_tokens)
        at = code_addresses(o, page_tokens, dim)
        for h in range(heads):
            for x, codes_at, scales_at in ((k[t, h], at[0], at[2]), (v[t, h], at[1], at[3])):
                codes, scales = quantise(x)
                out[page, h * block + codes_at] = codes[0::2] | codes[1::2] << 4
                out[page, h * block + scales_at] = scales
    return out


def read(pool, slots, heads: int, dim: int, page_tokens: int):
    """(k, v) [T, heads, D] fp64 of the slots; a negative or too large one gives zeros."""
    k, v = np.zeros((len(slots), heads, dim)), np.zeros((len(slots), heads, dim))
    block = page_tokens * (dim + 2 * (dim // 32))
    for t, slot in enumerate(slots):
        if not 0 <= slot < len(pool) * page_tokens:
            continue
        page, o = divmod(int(slot), page_tokens)
        at = code_addresses(o, page_tokens, dim)
        for h in range(heads):
            b = pool[page, h * block:(h + 1) * block]
            for x, codes_at, scales_at in ((k, at[0], at[2]), (v, at[1], at[3])):
                x[t, h] = values(np.stack((b[codes_at] & 15, b[codes_at] >> 4), -1).reshape(dim), b[scales_at])
    return k, v


# ---- attention
def attention(q, k, v, n_queries, scale: float, causal: bool = True):
    """q [T, heads, D] of the sequences one after the other, k[b], v[b] [keys, kv_heads, D] -> (out, weight) [T, heads, D]: the
    result, and the sum of p |v| that the error of a rounded probability is in proportion to.  A query without a key gives zeros."""
    q = np.asarray(q, np.float64)
    out, weight, at = np.zeros_like(q), np.zeros_like(q), 0
    for b, nq in enumerate(n_queries):
        keys, heads = k[b].shape[0], q.shape[1]
        for i in range(nq):
            n = max(0, keys - nq + i + 1) if causal else keys
            for h in range(heads if n else 0):
                kv = h // (heads // k[b].shape[1])
                s = scale * (k[b][:n, kv] @ q[at + i, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                out[at + i, h], weight[at + i, h] = p @ v[b][:n, kv], p @ np.abs(v[b][:n, kv])
        at += nq
    return out, weight
