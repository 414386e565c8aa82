"""Queries and keys normed and rotated, against the fp64 oracle.

Tolerances.  With u = 2^-24: a sum of D squares is off by at most D u of itself, its root by half that, and the few
products behind it by 8 u, so a normed value is off by (D/2 + 8) u of itself, the rotated one by that of |a| + |b|
(|cos|, |sin| <= 1); bf16 rows add half a unit of their last place, 2^-8 of the result (and of the error itself)."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2603_12118_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def table(n, half, theta=1e4):
    a = np.arange(n)[:, None] * theta ** (-np.arange(half) / half)
    return np.stack((np.cos(a), np.sin(a)), -1).astype(np.float32)


def check(got, x, cs, pos, sections, gain, eps, interleaved, dtype):
    D, half = x.shape[-1], int(sum(sections))
    want = O.norm_rope(x, cs, pos, sections, gain, eps, interleaved)
    y = np.abs(O.norm_rope(x, np.broadcast_to(np.array([1.0, 0.0]), cs.shape), pos, sections, gain, eps, interleaved))
    size = y.copy()
    size[..., :half] = size[..., half:2 * half] = y[..., :half] + y[..., half:2 * half]
    tol = (D / 2 + 8) * 2.0 ** -24 * size + 1e-37
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    g = got.double().cpu().numpy()
    assert g.shape == want.shape and np.isfinite(g).all()
    worst = (np.abs(g - want) / tol).max()
    assert worst <= 1, worst


def packed(rng, T, H, K, D, dtype, scale=1.0):
    """q, k as parts of one packed QKV tensor."""
    qkv = (torch.from_numpy(rng.standard_normal((T, H + 2 * K, D)) * scale)).to(TYPES[dtype]).to(DEV)
    return qkv, qkv[:, :H], qkv[:, H:H + K]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("T,H,K,D,sections,interleaved", [
    (1, 28, 4, 128, (16, 24, 24), False), (3, 1, 1, 64, (32,), False), (67, 8, 2, 64, (12, 10, 10), True), (130, 5, 3, 80, (8, 16, 16), False),
    (9, 4, 4, 96, (24, 24), False), (5, 3, 1, 256, (32, 48, 48), False), (33, 16, 16, 128, (24, 20, 20), True), (7, 2, 2, 16, (3, 5), False),
    (4, 6, 2, 128, (0, 16, 16), False), (2049, 2, 1, 48, (8,), False), (6, 40, 8, 128, (5, 3, 56), False), (2, 2, 1, 32, (6, 1, 1), True)])
def test_against_the_oracle(T, H, K, D, sections, interleaved, norm, dtype):
    rng = np.random.default_rng(T + D)
    qkv, q, k = packed(rng, T, H, K, D, dtype)
    before = qkv.clone()
    n, half = 50, sum(sections)
    cs = table(n, half)
    pos = rng.integers(0, n, (T, len(sections))).astype(np.int32)
    gains = [(1 + 0.2 * rng.standard_normal(D)).astype(np.float32) for _ in range(2)] if norm else [None, None]
    dg = [None if g is None else torch.from_numpy(g).to(DEV) for g in gains]
    flag = torch.zeros(1, dtype=torch.int32, device=DEV)
    args = dict(q_gain=dg[0], k_gain=dg[1], eps=1e-5, interleaved=interleaved, err_flag=flag)
    dcs, dpos = torch.from_numpy(cs).to(DEV), torch.from_numpy(pos).to(DEV)
    qo, ko = B.cs_qk_norm_rope(q, k, dcs, dpos, sections, **args)
    for got, x, gain in ((qo, q, gains[0]), (ko, k, gains[1])):
        check(got, x.double().cpu().numpy(), cs, pos, sections, gain, 1e-5, interleaved, dtype)
    assert torch.equal(qkv, before) and flag.item() == 0
    B.cs_qk_norm_rope(q, k, dcs, dpos, sections, q_out=q, k_out=k, **args)               # in place: the same bits, v untouched
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, H + K:], before[:, H + K:])


def test_far_positions_are_as_exact_as_the_table():
    rng = np.random.default_rng(0)
    _, q, k = packed(rng, 4, 2, 2, 128, "f32")
    cs = table(200000, 64)
    pos = np.array([[199999], [0], [131071], [65537]], np.int32)
    qo, ko = B.cs_qk_norm_rope(q, k, torch.from_numpy(cs).to(DEV), torch.from_numpy(pos).to(DEV), (64,))
    check(qo, q.double().cpu().numpy(), cs, pos, (64,), None, 0, False, "f32")


@pytest.mark.parametrize("scale", [1e-15, 1e15, 0.0])
def test_sizes_of_values(scale):
    # squares up to 1e30 and down to 1e-30, below eps; zeros give zeros
    rng = np.random.default_rng(1)
    _, q, k = packed(rng, 5, 2, 1, 64, "f32", scale)
    cs, pos = table(9, 32), rng.integers(0, 9, (5, 1)).astype(np.int32)
    g = torch.ones(64, device=DEV)
    qo, ko = B.cs_qk_norm_rope(q, k, torch.from_numpy(cs).to(DEV), torch.from_numpy(pos).to(DEV), (32,), q_gain=g, k_gain=g, eps=1e-6)
    check(qo, q.double().cpu().numpy(), cs, pos, (32,), np.ones(64), 1e-6, False, "f32")
    check(ko, k.double().cpu().numpy(), cs, pos, (32,), np.ones(64), 1e-6, False, "f32")


def test_positions_outside_the_table():
    rng = np.random.default_rng(2)
    _, q, k = packed(rng, 6, 3, 1, 64, "bf16")
    cs = table(10, 32)
    pos = np.array([[1, 2, 3], [10, 0, 0], [0, -1, 0], [9, 9, 9], [0, 0, 1 << 30], [0, 0, 0]], np.int32)
    flag = torch.zeros(1, dtype=torch.int32, device=DEV)
    qo, ko = torch.full((6, 3, 64), 3.0, dtype=torch.bfloat16, device=DEV), torch.full((6, 1, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    args = (torch.from_numpy(cs).to(DEV), torch.from_numpy(pos).to(DEV), (12, 10, 10))
    B.cs_qk_norm_rope(q, k, *args, q_out=qo, k_out=ko, err_flag=flag)
    assert flag.item() == 1
    for bad in (1, 2, 4):
        assert (qo[bad] == 3).all() and (ko[bad] == 3).all()
    ok = [0, 3, 5]
    check(qo[ok], q.double().cpu().numpy()[ok], cs, pos[ok], (12, 10, 10), None, 0, False, "bf16")
    B.cs_qk_norm_rope(q, k, *args)                                    # without a flag


def test_a_non_finite_head_stays_its_own():
    rng = np.random.default_rng(3)
    qkv, q, k = packed(rng, 3, 4, 2, 128, "bf16")
    cs, pos = torch.from_numpy(table(8, 64)).to(DEV), torch.tensor([[1], [2], [7]], dtype=torch.int32, device=DEV)
    g = torch.ones(128, device=DEV)
    clean, _ = B.cs_qk_norm_rope(q, k, cs, pos, (64,), q_gain=g, k_gain=g)
    q[1, 2, 5] = float("nan")
    got, _ = B.cs_qk_norm_rope(q, k, cs, pos, (64,), q_gain=g, k_gain=g)
    assert got[1, 2].isnan().all()
    got[1, 2] = clean[1, 2]
    assert torch.equal(got, clean)


def test_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(4)
    _, q, k = packed(rng, 12, 4, 2, 128, "bf16")
    cs, pos = torch.from_numpy(table(64, 64)).to(DEV), torch.zeros(12, 3, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    a, _ = B.cs_qk_norm_rope(q, k, cs, pos, (24, 20, 20), interleaved=True, stream=side)
    side.synchronize()
    qo, ko = torch.empty_like(a), torch.empty(12, 2, 128, dtype=a.dtype, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cs_qk_norm_rope(q, k, cs, pos, (24, 20, 20), interleaved=True, q_out=qo, k_out=ko)
    for i in range(4):
        pos.copy_(torch.randint(0, 64, (12, 3), device=DEV))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eq, ek = B.cs_qk_norm_rope(q, k, cs, pos, (24, 20, 20), interleaved=True)
        assert torch.equal(qo, eq) and torch.equal(ko, ek), i


def test_no_rows():
    _, q, k = packed(np.random.default_rng(5), 2, 4, 2, 64, "bf16")
    cs, pos = torch.from_numpy(table(4, 32)).to(DEV), torch.zeros(0, 1, dtype=torch.int32, device=DEV)
    qo, ko = B.cs_qk_norm_rope(q[:0], k[:0], cs, pos, (32,))
    assert qo.shape == (0, 4, 64) and ko.shape == (0, 2, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,sections", [(64, (16,)), (128, (8, 4, 4)), (80, (8, 16, 8)), (256, (32, 16, 16)), (48, (8,))])
def test_values_behind_the_rotary_part_pass_alone(D, sections, dtype):
    # whatever one of them is, an infinity or NaN, the others are not touched by it, and zeros keep their signs
    rng = np.random.default_rng(D)
    _, q, k = packed(rng, 4, 3, 2, D, dtype)
    rot = 2 * sum(sections)
    cs = torch.from_numpy(table(50, rot // 2)).to(DEV)
    pos = torch.from_numpy(rng.integers(0, 50, (4, len(sections))).astype(np.int32)).to(DEV)
    for x in (q, k):
        for i, value in enumerate((float("inf"), float("-inf"), float("nan"), 3e38)):
            x[i, 1, rot + 8] = value
            x[i, 0, rot + 1], x[i, 0, rot + 9] = -0.0, value
            x[i, 1, D - 1] = -0.0
    bits = torch.int16 if dtype == "bf16" else torch.int32
    for got, x in zip(B.cs_qk_norm_rope(q, k, cs, pos, sections), (q, k)):
        assert torch.equal(got[..., rot:].contiguous().view(bits), x[..., rot:].contiguous().view(bits))
        assert got[..., :rot].isfinite().all()
    # normed by an infinite mean: zeros, and NaN where the infinity was
    g = torch.ones(D, device=DEV)
    for got in B.cs_qk_norm_rope(q[:2], k[:2], cs, pos[:2], sections, q_gain=g, k_gain=g):
        want = torch.zeros_like(got)
        want[:, 1, rot + 8], want[:, 0, rot + 9] = float("nan"), float("nan")
        assert torch.equal(got[:, :2].isnan(), want[:, :2].isnan()) and not got[:, :2].nan_to_num().any()


# ---- waves that take several steps of heads (a wave takes HEADS = 8 heads of 128 or 16 of 64 a step; rows beyond 2048 workgroups of
# four share no row's heads out, and from 1024 on in fewer parts than steps): even and uneven parts, heads that end inside a step
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("T,H,K,D,sections,interleaved", [
    (8195, 28, 4, 128, (16, 24, 24), False),              # four steps, one part
    (4099, 40, 8, 128, (64,), False),                     # six steps, one part
    (2731, 40, 8, 128, (24, 20, 20), True),               # six steps, two parts
    (4093, 33, 2, 128, (10, 6, 16), False),               # five steps, two parts, the last step three heads; half of a head passes
    (2050, 16, 16, 128, (64,), False),                    # four steps, three parts
    (3001, 60, 10, 64, (32,), False),                     # five steps, two parts, the last step six heads
    (4100, 9, 2, 256, (32, 48, 48), False)])              # three steps of four heads, one part
def test_several_steps_a_wave(T, H, K, D, sections, interleaved, norm, dtype):
    HEADS = 64 // (4 if D <= 64 else 8 if D <= 128 else 16)
    steps, parts = -(-(H + K) // HEADS), max(1, 2048 // -(-T // 4))
    assert steps > parts
    rng = np.random.default_rng(T)
    qkv, q, k = packed(rng, T, H, K, D, dtype)
    n, half = 50, sum(sections)
    cs, pos = table(n, half), rng.integers(0, n, (T, len(sections))).astype(np.int32)
    gains = [(1 + 0.2 * rng.standard_normal(D)).astype(np.float32) for _ in range(2)] if norm else [None, None]
    dg = [None if g is None else torch.from_numpy(g).to(DEV) for g in gains]
    args = dict(q_gain=dg[0], k_gain=dg[1], eps=1e-5, interleaved=interleaved)
    dcs, dpos = torch.from_numpy(cs).to(DEV), torch.from_numpy(pos).to(DEV)
    before = qkv.clone()
    qo, ko = B.cs_qk_norm_rope(q, k, dcs, dpos, sections, **args)
    # (rows of every residue of a workgroup's four, at both ends and in between: the oracle is slow)
    some = np.unique(np.concatenate([np.arange(40), np.arange(T // 2, T // 2 + 40), np.arange(T - 40, T)]))
    for got, x, gain in ((qo, q, gains[0]), (ko, k, gains[1])):
        check(got[some], x[some].double().cpu().numpy(), cs, pos[some], sections, gain, 1e-5, interleaved, dtype)
    # ... and the rest against the same call on few rows at a time, where every wave has one step
    for a in range(0, T, 64):
        one = B.cs_qk_norm_rope(q[a:a + 64], k[a:a + 64], dcs, dpos[a:a + 64], sections, **args)
        assert torch.equal(qo[a:a + 64], one[0]) and torch.equal(ko[a:a + 64], one[1])
    assert torch.equal(qkv, before)
    B.cs_qk_norm_rope(q, k, dcs, dpos, sections, q_out=q, k_out=k, **args)
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, H + K:], before[:, H + K:])
