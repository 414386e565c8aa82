"""The measured operators of the rest of an LLM layer behind the attention over placed embeddings: the norms before and after a
block with its gate and residual scale, products of a few rows with weights laid out for it (4 bits with a scale for each 32 values,
or bf16), and a whole mixture-of-experts layer for a few tokens.

A state holds what a serving program has in hand before the call: hidden states, gains, the router, and the weights as it keeps
them.  Where ``own`` is false the operators run in their plain form, elementary torch operations in fp32 (the router's scores in
fp64, where two experts may lie close together) over weights kept as codes and scale bytes; where it is true, through the
framework's calls, over weights that it laid out once.

A case is a plain dict.  ``op`` is

* "norm"   ``rows`` tokens of ``width`` values: r = residual_scale residual + block_scale gate N(x), y = N(r), with N an RMSNorm or
           LayerNorm ("layer"); ``post`` whether x is normed, ``gate`` "none", "channel" (one row for all) or "row" (a row each),
           ``dtype`` of x, gate and y, ``residual`` that of the residual rows;
* "linear" ``rows`` tokens against a matrix of ``n`` rows of ``k`` values, ``format`` "e2m1" or "bf16", ``bias``, ``out`` the type of y;
* "moe"    ``rows`` tokens, the last ``idle`` of them padding rows of a recorded step; ``hidden``, ``inter``, ``experts``, ``top``,
           ``shared`` experts that every token takes, ``score`` "softmax" or "sigmoid" (with a bias that steers the choice),
           ``format`` of the experts.

A group of 32 values along k has one power of two (a byte, exponent + 127) and 32 codes of 4 bits (sign, and an index into
0 .5 1 1.5 2 3 4 6), as in the cache.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
GROUP = 32                  # values that share a scale
EPS = 1e-6
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ---------------------------------------------------------------------------------------------------
def _norm(rows, width, norm="rms", post=True, gate="none", dtype="bf16", residual="bf16"):
    return {"op": "norm", "rows": rows, "width": width, "norm": norm, "post": post, "gate": gate, "dtype": dtype, "residual": residual}


def _linear(rows, n, k, format="e2m1", bias=False, out="bf16"):
    return {"op": "linear", "rows": rows, "n": n, "k": k, "format": format, "bias": bias, "out": out}


def _moe(rows, hidden, inter, experts, top, shared=0, score="softmax", format="e2m1", idle=0):
    return {"op": "moe", "rows": rows, "hidden": hidden, "inter": inter, "experts": experts, "top": top, "shared": shared,
            "score": score, "format": format, "idle": idle}


def listed():
    return [
        # one generated token between two blocks of a layer of 3584: latency alone
        {"name": "norm_token", **_norm(1, 3584)},
        # an odd number of rows of a tower's width, LayerNorm with a learned scale on each channel, all in fp32
        {"name": "norm_1125_f32", **_norm(1125, 1280, norm="layer", gate="channel", dtype="f32", residual="f32")},
        # a packed prompt batch, a gate for each row, the residual stream kept in fp32
        {"name": "norm_16384", **_norm(16384, 3584, gate="row", residual="f32")},
        # queries, keys and values of one generated token
        {"name": "linear_token_qkv", **_linear(1, 4608, 3584, bias=True)},
        # gate and up of one generated token in a dense layer, four times as wide as the hidden states
        {"name": "linear_token_up", **_linear(1, 28672, 3584)},
        # the output projection of eight sequences' tokens, weights not quantised
        {"name": "linear_8_bf16", **_linear(8, 3584, 3584, format="bf16")},
        # the way back down of a decode batch, an odd number of sequences
        {"name": "linear_45_down", **_linear(45, 3584, 14336, out="f32")},
        # gate and up of a chunk of a prompt
        {"name": "linear_256_up", **_linear(256, 28672, 3584)},
        # one generated token through many small experts
        {"name": "moe_token", **_moe(1, 2048, 768, 128, 8)},
        # eight sequences' tokens, few large experts in bf16, one of them every token's
        {"name": "moe_8_bf16", **_moe(8, 3584, 1280, 16, 2, shared=1, score="sigmoid", format="bf16")},
        # a decode batch padded with idle rows as a recorded step pads it
        {"name": "moe_48", **_moe(48, 2048, 768, 128, 8, idle=3)},
        # a chunk of a prompt
        {"name": "moe_512", **_moe(512, 2048, 768, 128, 8)},
    ]


# hidden, inter, experts, top, shared
_LAYERS = ((2048, 768, 128, 8, 0), (3584, 1280, 16, 2, 1), (1024, 512, 64, 6, 2), (2560, 1024, 32, 4, 0), (1056, 352, 24, 3, 0), (512, 96, 200, 10, 0))


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "linear", "linear", "linear", "moe", "moe", "moe"])
    if op == "norm":
        width = 8 * _log_int(rng, 8, 2048)
        rows = min(_log_int(rng, 1, 16384), 16384 * 3584 // (2 * width))
        dtype = rng.choice(["bf16", "bf16", "f32"])
        return _norm(rows, width, rng.choice(["rms", "rms", "layer"]), rng.random() < 0.7, rng.choice(["none", "channel", "row"]), dtype,
                     "f32" if dtype == "f32" else rng.choice(["bf16", "f32"]))
    if op == "linear":
        format = rng.choice(["e2m1", "e2m1", "e2m1", "bf16"])
        k = 32 * _log_int(rng, 2, 448)
        n = min(_log_int(rng, 48, 28672), 28672 * 3584 // k if format == "e2m1" else 28672 * 3584 // (4 * k))
        return _linear(_log_int(rng, 1, 256), n, k, format, rng.random() < 0.5, rng.choice(["bf16", "bf16", "f32"]))
    hidden, inter, experts, top, shared = rng.choice(_LAYERS)
    rows = _log_int(rng, 1, 512)
    if hidden * inter * experts > 64 << 20 and rng.random() < 0.5:
        rows = _log_int(rng, 1, 64)
    return _moe(rows, hidden, inter, experts, top, shared, rng.choice(["softmax", "softmax", "sigmoid"]),
                "bf16" if rng.random() < 0.3 and hidden * inter * experts <= 96 << 20 else "e2m1", rows // 16 * rng.randint(0, 2))


# ---- weights as they are held ----------------------------------------------------------------------------------
def _quantise(w):
    """[..., k] bf16 -> (bytes of two codes [..., k / 2], scale bytes [..., k / 32])."""
    x = w.float().view(*w.shape[:-1], -1, GROUP)
    byte = ((x.abs().amax(-1).view(torch.int32) + 0x200000 >> 23) - 2).clamp(2, 252)
    y = x * (254 - byte << 23).view(torch.float32)[..., None]
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6.0)
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) + 8 * (y < 0).to(torch.uint8)
    code = code.flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], byte.to(torch.uint8)


def _values(codes, scales):
    """The reverse of _quantise, fp32."""
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=codes.device)
    y = level[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    power = (scales.int() << 23).view(torch.float32)
    return (y.view(*scales.shape, GROUP) * power[..., None]).flatten(-2)


def _keep(w, format):
    """What a program keeps of weights [matrices, n, k] bf16."""
    if own:
        from paper_2603_12118_amd import binding as B
        return B.cs_weights_pack(w, format)
    if format == "bf16":
        return w
    parts = [_quantise(p) for p in w.split(max(1, (64 << 20) // w[0].numel()))]
    return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


def _matrix(kept, e):
    """Matrix e of plain weights, fp32."""
    return kept[e].float() if isinstance(kept, torch.Tensor) else _values(kept[0][e], kept[1][e])


# ---- states ----------------------------------------------------------------------------------------------------
class _State:
    pass


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _inputs(case, seed):
    """Everything but the weights as they are kept: those in bf16, [matrices, n, k]."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    s = _State()
    s.case = case
    T = case["rows"]
    if case["op"] == "norm":
        W, dtype = case["width"], TYPES[case["dtype"]]
        # a residual stream of a few loud channels, and what a block adds to it
        s.residual = (_randn(gen, T, W) * (1 + 20 * (torch.rand(W, generator=gen, device=DEV) < 0.01))).to(TYPES[case["residual"]])
        s.x = (0.5 * _randn(gen, T, W) + 0.1).to(dtype)
        s.gate = {"none": None, "channel": (0.1 + 0.02 * _randn(gen, W)).to(dtype), "row": None}[case["gate"]]
        if case["gate"] == "row":
            s.gate = torch.sigmoid(_randn(gen, T, W)).to(dtype)
        s.pre_gain, s.post_gain = (1 + 0.1 * _randn(gen, W) for _ in range(2))
        s.pre_bias, s.post_bias = (0.1 * _randn(gen, W) if case["norm"] == "layer" else None for _ in range(2))
        if not case["post"]:
            s.post_gain = s.post_bias = None
        s.scales = (0.5 + float(torch.rand(1, generator=gen, device=DEV)), 0.5 + float(torch.rand(1, generator=gen, device=DEV)))
    elif case["op"] == "linear":
        s.x = _randn(gen, T, case["k"]).bfloat16()
        s.w = (_randn(gen, 1, case["n"], case["k"]) * case["k"] ** -0.5).bfloat16()
        s.bias = 0.1 * _randn(gen, case["n"]) if case["bias"] else None
    else:
        H, I, E, S = case["hidden"], case["inter"], case["experts"], case["shared"]
        s.x = _randn(gen, T, H).bfloat16()
        s.router = (_randn(gen, E, H) * H ** -0.5).bfloat16()
        s.choice_bias = 0.05 * _randn(gen, E) if case["score"] == "sigmoid" else None
        s.live = torch.arange(T, device=DEV) < T - case["idle"] if case["idle"] else None
        s.up = torch.empty(E + S, 2 * I, H, device=DEV, dtype=torch.bfloat16).normal_(0, H ** -0.5, generator=gen)
        s.down = torch.empty(E + S, H, I, device=DEV, dtype=torch.bfloat16).normal_(0, I ** -0.5, generator=gen)
        s.scale = 1.0 if case["score"] == "softmax" else 2.5
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "linear":
        s.w = _keep(s.w, case["format"])
    elif case["op"] == "moe":
        s.up, s.down = _keep(s.up, case["format"]), _keep(s.down, case["format"])
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------
def _plain_n(x, kind, gain, bias):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
    return y if bias is None else y + bias


def _plain_norm(s):
    case = s.case
    z = s.x.float()
    if case["post"]:
        z = _plain_n(z, case["norm"], s.post_gain, s.post_bias)
    if s.gate is not None:
        z = z * s.gate.float()
    r = s.scales[0] * s.residual.float() + s.scales[1] * z
    y = _plain_n(r, case["norm"], s.pre_gain, s.pre_bias)
    return {"residual": r.to(s.residual.dtype), "y": y.to(s.x.dtype)}


def _plain_route(s):
    """Experts [T, top] and their weights [T, top] fp64, the best first; a row that is not live has weights of zero."""
    case, k = s.case, s.case["top"]
    logits = s.x.double() @ s.router.double().t()
    score = torch.softmax(logits, -1) if case["score"] == "softmax" else torch.sigmoid(logits)
    choice = logits if s.choice_bias is None else score + s.choice_bias.double()
    experts = torch.sort(choice, dim=-1, descending=True, stable=True)[1][:, :k]
    weights = score.gather(1, experts)
    weights = weights / weights.sum(-1, keepdim=True) * s.scale
    if s.live is not None:
        experts, weights = torch.where(s.live[:, None], experts, -1), weights * s.live[:, None]
    return experts, weights


def _plain_moe(s):
    case = s.case
    E, I = case["experts"], case["inter"]
    experts, weights = _plain_route(s)
    x, w32 = s.x.float(), weights.float()
    y = torch.zeros_like(x)
    for e in range(E + case["shared"]):
        up = x @ _matrix(s.up, e).t()
        g, u = up[:, :I], up[:, I:]
        h = g / (1 + torch.exp(-g)) * u
        if e < E:
            share = (w32 * (experts == e)).sum(-1, keepdim=True)
        else:
            share = torch.ones_like(w32[:, :1]) if s.live is None else s.live[:, None].float()
        y += share * (h @ _matrix(s.down, e).t())
    return {"y": y.to(s.x.dtype), "experts": experts.int(), "weights": w32}


def run(state):
    s, case = state, state.case
    if own:
        from paper_2603_12118_amd import binding as B
        if case["op"] == "norm":
            r, y = B.cs_norm_residual(s.x, s.residual, pre_gain=s.pre_gain, pre_bias=s.pre_bias, post_gain=s.post_gain, post_bias=s.post_bias,
                                      gate=s.gate, residual_scale=s.scales[0], block_scale=s.scales[1], norm=case["norm"], eps=EPS)
            return {"residual": r, "y": y}
        if case["op"] == "linear":
            return B.cs_linear_packed(s.x, s.w, bias=s.bias, dtype=TYPES[case["out"]])
        y, experts, weights = B.cs_moe(s.x, s.router, s.up, s.down, case["top"], score=case["score"], renormalise=True, scale=s.scale,
                                       choice_bias=s.choice_bias, live=s.live)
        return {"y": y, "experts": experts, "weights": weights}
    if case["op"] == "norm":
        return _plain_norm(s)
    if case["op"] == "linear":
        y = s.x.float() @ _matrix(s.w, 0).t()
        return (y if s.bias is None else y + s.bias).to(TYPES[case["out"]])
    return _plain_moe(s)


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def _held_bytes(case, values):
    return values * (0.5 + 1 / GROUP) if case["format"] == "e2m1" else 2.0 * values


def work(case):
    T = case["rows"]
    if case["op"] == "norm":
        size, rsize, W = (2 if case["dtype"] == "bf16" else 4), (2 if case["residual"] == "bf16" else 4), case["width"]
        vectors = 4 * W * (1 + case["post"]) * (2 if case["norm"] == "layer" else 1) + (size * W if case["gate"] == "channel" else 0)
        return {"bytes": float(T * W * (2 * size + 2 * rsize + (size if case["gate"] == "row" else 0)) + vectors), "flops": float(14 * T * W)}
    if case["op"] == "linear":
        n, k = case["n"], case["k"]
        return {"bytes": float(_held_bytes(case, n * k) + 2 * T * k + T * n * (2 if case["out"] == "bf16" else 4) + (4 * n if case["bias"] else 0)),
                "flops": float(2 * T * n * k)}
    H, I, E, k, S = case["hidden"], case["inter"], case["experts"], case["top"], case["shared"]
    T -= case["idle"]
    used = E * (1 - (1 - k / E) ** T) + S           # experts that some token takes, where all are as likely
    return {"bytes": float(_held_bytes(case, used * 3 * H * I) + 2 * E * H + 2 * T * H + 2 * case["rows"] * H + 8 * case["rows"] * k),
            "flops": float(6 * T * (k + S) * H * I + 2 * T * E * H)}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------
def _two_to(e):
    """2^e in fp64, e a tensor of whole numbers."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _exact_held(x, format):
    """The values that a matrix [n, k] is held as, fp64: per 32 of them, the nearest level at the group's power of two."""
    x = x.double()
    if format == "bf16":
        return x
    x = x.reshape(x.shape[0], -1, 32)
    top = x.abs().amax(-1, keepdim=True)
    mantissa, exponent = torch.frexp(top)           # top = mantissa 2^exponent, 1/2 <= mantissa < 1
    e = (exponent - 3 + (mantissa >= 0.875)).clamp(-125, 125)
    e = torch.where(top == 0, -125, e)
    y = x.abs() * _two_to(-e)
    held = torch.zeros_like(y)
    for n, (lo, hi) in enumerate(zip(LEVELS[:-1], LEVELS[1:])):
        mid = (lo + hi) / 2
        held = torch.where((y > mid) | ((y == mid) & (n % 2 == 1)), hi, held)        # a tie goes to the even code
    return (held * _two_to(e) * x.sign()).flatten(1)


def _exact_n(x, kind, gain, bias):
    if kind == "layer":
        var, mean = torch.var_mean(x, dim=-1, correction=0, keepdim=True)
        x = (x - mean) * torch.rsqrt(var + EPS)
    else:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    x = x * gain.double()
    return x + bias.double() if bias is not None else x


def exact(case, seed):
    s = _inputs(case, seed)
    x = s.x.double()
    if case["op"] == "norm":
        z = _exact_n(x, case["norm"], s.post_gain, s.post_bias) if s.post_gain is not None else x
        z = z * s.gate.double() if s.gate is not None else z
        r = torch.add(s.residual.double() * s.scales[0], z, alpha=s.scales[1])
        return {"residual": r, "y": _exact_n(r, case["norm"], s.pre_gain, s.pre_bias)}
    if case["op"] == "linear":
        y = torch.cat([x @ _exact_held(w, case["format"]).T for w in s.w[0].split(8192)], -1)
        return y + s.bias.double() if s.bias is not None else y
    E, I, k, T = case["experts"], case["inter"], case["top"], case["rows"]
    logits = x @ s.router.double().T
    if case["score"] == "softmax":
        score = torch.exp(logits - logits.logsumexp(-1, keepdim=True))
    else:
        score = 1 / (1 + torch.exp(-logits))
    choice = logits.clone() if s.choice_bias is None else score + s.choice_bias.double()
    alive = torch.ones(T, dtype=torch.bool, device=DEV) if s.live is None else s.live
    experts = torch.full((T, k), -1, dtype=torch.long, device=DEV)
    weights = torch.zeros(T, k, dtype=torch.float64, device=DEV)
    for i in range(k):                              # the largest that is left, the lowest number of equal ones
        best = choice == choice.amax(-1, keepdim=True)
        experts[:, i] = torch.where(best, torch.arange(E, device=DEV), E).amin(-1)
        choice.scatter_(1, experts[:, i:i + 1], -math.inf)
        weights[:, i] = score.gather(1, experts[:, i:i + 1])[:, 0]
    weights *= (s.scale * alive / weights.sum(-1))[:, None]
    experts[~alive] = -1
    y = torch.zeros_like(x)
    for e in range(E + case["shared"]):
        rows, at = (experts == e).nonzero(as_tuple=True) if e < E else (alive.nonzero()[:, 0], None)
        if not len(rows):
            continue
        up = x[rows] @ _exact_held(s.up[e], case["format"]).T
        h = up[:, :I] * torch.sigmoid(up[:, :I]) * up[:, I:]
        out = h @ _exact_held(s.down[e], case["format"]).T
        y[rows] += out if at is None else weights[rows, at][:, None] * out
    return {"y": y, "experts": experts, "weights": weights}
