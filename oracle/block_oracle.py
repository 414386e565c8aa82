"""CPU oracle of the LLM task's layer behind its attention: norms around a block, products with packed weights, experts.

Written from the definitions in include/cornenc.h in numpy fp64, with the bounds that the arithmetic of the calls allows beside the
values (fp32 sums, the roundings that the definitions name); test infrastructure only.  What 4-bit weights are held as is the cache's
format (cache_oracle.held).
"""
from __future__ import annotations

import numpy as np

from oracle import cache_oracle

U = 2.0 ** -24                                   # half a step of fp32
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}    # half a step, relative


def norm(x, kind, gain, bias, eps):
    x = np.asarray(x, np.float64)
    if kind == "layer":
        x = x - x.mean(-1, keepdims=True)
    s = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    y = x * s * gain
    return y if bias is None else y + bias, s


def norm_residual(x, residual, pre_gain, pre_bias=None, post_gain=None, post_bias=None, gate=None, residual_scale=1.0, block_scale=1.0,
                  kind="rms", eps=1e-6, r_type="bf16", y_type="bf16"):
    """(r, y, largest error of r, largest error of y).

    The calls sum a row's squares and values in at most 32 steps a lane and 16 joining them, so that a sum of positive terms is off by 48 U of
    itself, and a root, a quotient and a few products add 10: 64 U of what enters a value bounds it, the mean of the magnitudes included
    where a mean is taken away.  An error d of r reaches y by r itself, by the mean and by the root of the mean square."""
    x, residual = np.asarray(x, np.float64), np.asarray(residual, np.float64)
    z, mag = x, np.abs(x)
    if post_gain is not None:
        z, s = norm(x, kind, post_gain, post_bias, eps)
        mag = (np.abs(x) + (mag.mean(-1, keepdims=True) if kind == "layer" else 0)) * s * np.abs(post_gain) * (1 + (s * np.abs(x)).mean(-1, keepdims=True))
        mag = mag + (0 if post_bias is None else np.abs(post_bias))
    if gate is not None:
        z, mag = z * gate, mag * np.abs(gate)
    r = residual_scale * residual + block_scale * z
    d = 64 * U * (np.abs(residual_scale * residual) + np.abs(block_scale) * mag)
    y, s = norm(r, kind, pre_gain, pre_bias, eps)
    c = r - r.mean(-1, keepdims=True) if kind == "layer" else r
    dc = d + d.mean(-1, keepdims=True) + 64 * U * (np.abs(r) + np.abs(r).mean(-1, keepdims=True))
    dy = np.abs(pre_gain) * s * (dc + np.abs(c) * s * np.sqrt((dc * dc).mean(-1, keepdims=True))) + 64 * U * np.abs(y)
    if pre_bias is not None:
        dy = dy + 64 * U * np.abs(pre_bias)
    return r, y, 1.01 * d + HALF[r_type] * np.abs(r), 1.01 * dy + HALF[y_type] * (np.abs(y) + dy)


def held(w, format):
    """The values weights [.., k] are held as; bf16 weights are given as such."""
    w = np.asarray(w, np.float64)
    return w if format == "bf16" else cache_oracle.held(w)


def product(x, w, dx=None):
    """x w^T and its largest error: fp32 sums of k products in any order, and errors dx of x."""
    a = np.abs(x) @ np.abs(w).T
    d = (w.shape[1] + 64) * U * a
    return x @ w.T, d if dx is None else d + dx @ np.abs(w).T


def linear(x, w, bias=None, out_type="bf16"):
    y, d = product(np.asarray(x, np.float64), np.asarray(w, np.float64))
    if bias is not None:
        y = y + bias
        d = d + 2 * U * np.abs(y)
    return y, d + HALF[out_type] * (np.abs(y) + d)


def route(x, router, top, score="softmax", renormalise=True, scale=1.0, choice_bias=None, live=None):
    """experts [T, top] and weights [T, top] (-1 and 0 of rows that are not live)."""
    logits = np.asarray(x, np.float64) @ np.asarray(router, np.float64).T
    if score == "softmax":
        with np.errstate(invalid="ignore"):
            e = np.exp(logits - np.nanmax(np.where(np.isnan(logits), -np.inf, logits), -1, keepdims=True))
        p = e / e.sum(-1, keepdims=True)
    else:
        p = 1 / (1 + np.exp(-logits))
    choice = logits if choice_bias is None else p + np.asarray(choice_bias, np.float64)
    key = np.where(np.isnan(choice), -np.inf, choice)
    # (a NaN is below every number, -inf among them)
    experts = np.stack([np.lexsort((np.arange(key.shape[1]), -k, np.isnan(c))) for k, c in zip(key, choice)])[:, :top] if len(key) else np.zeros((0, top), int)
    weights = np.take_along_axis(p, experts, -1)
    if renormalise:
        weights = weights / weights.sum(-1, keepdims=True)
    weights = weights * scale
    if live is not None:
        dead = ~np.asarray(live, bool)
        experts, weights = np.where(dead[:, None], -1, experts), np.where(dead[:, None], 0.0, weights)
    return experts, weights


def expert(x, up, down):
    """down (silu(g) * u) of rows x, with the largest error: fp32 sums, exponentials off by 2^-17 at most (|g| up to 80 steps of 2^-24 and a
    few), silu(g) * u rounded to bf16, |silu'| < 1.1."""
    inter = up.shape[0] // 2
    p, dp = product(x, up)
    g, u, dg, du = p[:, :inter], p[:, inter:], dp[:, :inter], dp[:, inter:]
    a = g / (1 + np.exp(-g))
    h = a * u
    dh = 1.1 * dg * (np.abs(u) + du) + np.abs(a) * du + 2.0 ** -17 * np.abs(h)
    dh = dh + HALF["bf16"] * (np.abs(h) + dh) + 2.0 ** -133       # (and a step of the smallest numbers)
    y, d = product(h, down, dh)
    return y, d


def moe(x, router, up, down, top, **kw):
    """(y, experts, weights, largest error of y); up [matrices, 2 inter, hidden] and down [matrices, hidden, inter] as they are held."""
    x = np.asarray(x, np.float64)
    experts, weights = route(x, router, top, **kw)
    live = np.ones(len(x), bool) if kw.get("live") is None else np.asarray(kw["live"], bool)
    y, d = np.zeros((len(x), down.shape[1])), np.zeros((len(x), down.shape[1]))
    for e in range(len(up)):
        if e < len(router):
            rows, at = np.nonzero(experts == e)
            w = weights[rows, at][:, None]
        else:
            rows = np.nonzero(live)[0]
            w = np.ones((len(rows), 1))
        if len(rows):
            out, do = expert(x[rows], up[e], down[e])
            y[rows] += w * out
            d[rows] += np.abs(w) * (do + 64 * U * np.abs(out))
    return y, experts, weights, d + HALF["bf16"] * (np.abs(y) + d)
