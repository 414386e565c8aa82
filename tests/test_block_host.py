"""The calls of the layer behind the attention without a GPU: the CPU oracle against brute force, and what the calls refuse before
anything is enqueued."""
import ctypes as C

import numpy as np
import pytest

from oracle import block_oracle as O
from paper_2603_12118_amd import binding as B

INV, WS, UNS = B.CS_ERR_INVALID_ARG, B.CS_ERR_WORKSPACE, B.CS_ERR_UNSUPPORTED


# ---- the oracle
def test_norm_residual_by_hand():
    x, res = np.array([[3.0, 4.0]]), np.array([[1.0, 1.0]])
    r, y, dr, dy = O.norm_residual(x, res, np.array([1.0, 2.0]), post_gain=np.array([2.0, 1.0]), gate=np.array([0.5, 2.0]), residual_scale=2.0,
                                   block_scale=3.0, eps=0.0)
    n = np.sqrt(12.5)
    want = np.array([2 + 3 * (3 / n * 2 * 0.5), 2 + 3 * (4 / n * 2)])
    assert np.allclose(r, want) and np.allclose(y, want / np.sqrt((want ** 2).mean()) * [1, 2])
    assert (dr >= 2.0 ** -8 * np.abs(r)).all() and (dr < 2.01 * 2.0 ** -8 * np.abs(r)).all() and (dy < 2.01 * 2.0 ** -8 * np.abs(y)).all()
    _, y, _, _ = O.norm_residual(x, res, np.ones(2), np.array([5.0, 6.0]), kind="layer", eps=0.0)
    assert np.allclose(y, [[4.0, 7.0]])


def test_route_by_hand():
    x = np.eye(3)
    router = np.array([[1.0, 0, 0], [3, 0, -1], [3, 0, 2], [2, 0, -np.inf]])
    e, w = O.route(x[:2] + [0, 0, -1e-300], router[:, :2] @ np.eye(2, 3), 3)
    assert list(e[0]) == [1, 2, 3] and list(e[1]) == [0, 1, 2]
    assert np.allclose(w[0], np.exp([3, 3, 2]) / np.exp([3, 3, 2]).sum())
    with np.errstate(invalid="ignore"):
        e, w = O.route(x[2:], router, 4)                 # 0, -1, 2 and 2 * 0 - inf
    assert list(e[0]) == [2, 0, 1, 3]
    router[3, 2] = np.nan
    e, w = O.route(x[2:], router, 4)
    assert list(e[0]) == [2, 0, 1, 3] and np.isnan(w).all()
    e, w = O.route(x[:2], router[:3], 2, score="sigmoid", choice_bias=[0, -1, 0], scale=2.0, renormalise=False, live=[1, 0])
    assert list(e[0]) == [2, 0] and np.allclose(w[0], 2 / (1 + np.exp([-3.0, -1.0]))) and list(e[1]) == [-1, -1] and not w[1].any()


def test_moe_is_the_sum_over_rows_and_experts():
    rng = np.random.default_rng(0)
    x, router = rng.standard_normal((4, 6)), rng.standard_normal((3, 6))
    up, down = rng.standard_normal((4, 10, 6)), rng.standard_normal((4, 6, 5))
    y, e, w, d = O.moe(x, router, up, down, 2)
    for t in range(4):
        want = np.zeros(6)
        for i, s in list(zip(e[t], w[t])) + [(3, 1.0)]:
            g, u = (up[i] @ x[t])[:5], (up[i] @ x[t])[5:]
            want += s * (down[i] @ (g / (1 + np.exp(-g)) * u))
        assert np.allclose(y[t], want)
    assert (d > 0).all() and (d < 0.05 * sum(np.abs(x) @ np.abs(u).T @ np.ones((10, 6)) for u in up) * np.abs(x @ up[0].T).max() * np.abs(down).max()).all()


# ---- refusals: pointers here are plain numbers, nothing is enqueued
def norm_status(x=256, x_row=64, res=512, res_row=64, og=0, ob=0, pg=1024, pb=0, r=2048, r_row=64, y=4096, y_row=64, n=3, **kw):
    d = dict(struct_size=C.sizeof(B.cs_norm_config), norm=0, width=64, dtype=B.CS_BF16, residual_dtype=B.CS_F32, gate=0, eps=1e-6, residual_scale=1.0,
             block_scale=1.0) | kw
    return B.lib().cs_norm_residual(C.byref(B.cs_norm_config(**d)), x, x_row, res, res_row, 0, 64, og, ob, pg, pb, r, r_row, y, y_row, n, None)


def test_norm_residual_refusals():
    assert B.lib().cs_norm_residual(None, *([256, 64] * 2), 0, 0, 0, 0, 64, 0, 256, 64, 256, 64, 1, None) == INV
    assert norm_status(struct_size=4) == INV and norm_status(norm=2) == INV and norm_status(dtype=2) == INV and norm_status(residual_dtype=-1) == INV
    assert norm_status(width=0) == INV and norm_status(width=-8) == INV and norm_status(width=60) == UNS
    assert norm_status(width=16392, x_row=16392, res_row=16392, r_row=16392, y_row=16392) == UNS
    nan, inf = float("nan"), float("inf")
    assert norm_status(eps=-1.0) == INV and norm_status(eps=nan) == INV and norm_status(residual_scale=inf) == INV and norm_status(block_scale=nan) == INV
    assert norm_status(n=-1) == INV and norm_status(n=1 << 31) == UNS and norm_status(n=0) == 0 and norm_status(n=0, x=0, y=0) == 0
    for name in ("x", "res", "r", "y"):
        assert norm_status(**{name: 0}) == INV and norm_status(**{name: 264}) == INV
        assert norm_status(**{name + "_row": 63}) == INV and norm_status(**{name + "_row": 1 << 41}) == INV
    assert norm_status(x_row=68) == UNS and norm_status(res_row=66) == UNS
    assert norm_status(gate=3) == INV and norm_status(pg=0) == INV and norm_status(pg=8) == INV and norm_status(ob=64) == INV and norm_status(pb=4) == INV
    assert "cs_norm_residual" in B.last_error()
    c = dict(struct_size=C.sizeof(B.cs_norm_config), norm=0, width=64, dtype=1, residual_dtype=0, gate=2, eps=0, residual_scale=1, block_scale=1)
    call = lambda g, row: B.lib().cs_norm_residual(C.byref(B.cs_norm_config(**c)), 256, 64, 512, 64, g, row, 0, 0, 1024, 0, 2048, 64, 4096, 64, 3, None)
    assert call(0, 64) == INV and call(24, 64) == INV and call(256, 56) == INV and call(256, 68) == UNS


def weights(**kw):
    d = dict(struct_size=C.sizeof(B.cs_weights_config), format=0, matrices=1, n=48, k=64) | kw
    return B.cs_weights_config(**d)


@pytest.mark.parametrize("read", [False, True])
def test_weights_refusals(read):
    def st(c=None, w=256, row=64, matrix=4096, dtype=B.CS_BF16, packed=512, err=0):
        c = weights() if c is None else c
        if read:
            return B.lib().cs_weights_read(C.byref(c), packed, w, row, matrix, dtype, None)
        return B.lib().cs_weights_pack(C.byref(c), w, row, matrix, dtype, packed, err, None)
    assert st(weights(struct_size=4)) == INV and st(weights(format=2)) == INV and st(weights(n=0)) == INV and st(weights(matrices=-1)) == INV
    assert st(weights(k=48)) == UNS and st(weights(n=(1 << 24) + 1)) == UNS and st(weights(matrices=1 << 20, n=1 << 24, k=1 << 24)) == UNS
    assert st(dtype=5) == INV and st(w=0) == INV and st(w=8) == INV and st(row=56) == INV and st(row=68) == UNS
    assert st(packed=0) == INV and st(packed=24) == INV and st(matrix=-64) == INV and st(weights(matrices=2), matrix=4100) == UNS
    assert st(matrix=0, w=0) == INV
    if read:
        assert st(weights(matrices=2), matrix=47 * 64 + 56) == INV and "overlap" in B.last_error()
    else:
        assert st(err=2) == INV


def test_weights_query():
    assert B.cs_weights_query("e2m1", 48, 64) == 3 * 1088 and B.cs_weights_query("e2m1", 33, 160, 7) == 7 * 3 * 2 * 1088
    assert B.cs_weights_query("bf16", 48, 96) == 48 * 96 * 2
    assert B.cs_weights_query("e2m1", 65536, 65536, 1000) == 1000 * 65536 * 65536 * 17 // 32           # past 32 bits
    with pytest.raises(ValueError):
        B.cs_weights_query("int4", 48, 64)
    assert B.lib().cs_weights_query(C.byref(weights()), None) == INV and B.lib().cs_weights_query(None, C.byref(C.c_size_t())) == INV


def test_linear_refusals():
    L = B.lib()

    def st(c=None, packed=256, x=512, x_row=64, bias=0, out=1024, out_row=48, dtype=B.CS_BF16, n=3, ws=2048, ws_bytes=1 << 40):
        return L.cs_linear_packed(C.byref(weights() if c is None else c), packed, x, x_row, bias, out, out_row, dtype, n, ws, ws_bytes, None)
    assert st(weights(struct_size=0)) == INV and st(weights(matrices=2)) == INV and st(weights(k=40)) == UNS
    assert st(n=-1) == INV and st(n=1 << 31) == UNS and st(n=0) == 0 and st(n=0, x=0, out=0, ws=0) == 0
    assert st(packed=0) == INV and st(packed=8) == INV and st(x=0) == INV and st(x=520) == INV and st(x_row=56) == INV and st(x_row=68) == UNS
    assert st(x_row=(1 << 22) + 8) == UNS
    assert st(out=0) == INV and st(out=1025) == INV and st(out=1026, dtype=B.CS_F32) == INV and st(out_row=47) == INV and st(dtype=3) == INV and st(bias=2) == INV
    need = C.c_size_t()
    c = weights(k=65536)
    assert L.cs_linear_packed_query(C.byref(c), 40, C.byref(need)) == 0 and need.value > 0
    assert st(c, x_row=65536, n=40, ws_bytes=need.value - 1) == WS and st(c, x_row=65536, n=40, ws=0) == INV and st(c, x_row=65536, n=40, ws=8) == INV
    assert L.cs_linear_packed_query(C.byref(c), 40, None) == INV and L.cs_linear_packed_query(C.byref(weights(k=1)), 40, C.byref(need)) == UNS
    assert L.cs_linear_packed_query(C.byref(weights(n=1 << 24)), (1 << 31) - 1, C.byref(need)) == UNS


def moe(**kw):
    d = dict(struct_size=C.sizeof(B.cs_moe_config), format=0, hidden=64, inter=32, n_experts=8, n_shared=1, top=2, score=0, renormalise=1, scale=1.0) | kw
    return B.cs_moe_config(**d)


def test_moe_refusals():
    L = B.lib()

    def st(c=None, x=256, x_row=64, router=512, bias=0, live=0, up=1024, down=2048, y=4096, y_row=64, experts=16, w=32, n=3, ws=8192, ws_bytes=1 << 40):
        return L.cs_moe(C.byref(moe() if c is None else c), x, x_row, router, bias, live, up, down, y, y_row, experts, w, n, ws, ws_bytes, None)
    assert L.cs_moe(None, 256, 64, 512, 0, 0, 1024, 2048, 4096, 64, 16, 32, 3, 8192, 1 << 40, None) == INV
    assert st(moe(struct_size=1)) == INV and st(moe(format=-1)) == INV and st(moe(score=2)) == INV and st(moe(renormalise=2)) == INV
    assert st(moe(scale=float("nan"))) == INV
    for name in ("hidden", "inter", "n_experts", "top"):
        assert st(moe(**{name: 0})) == INV
    assert st(moe(n_shared=-1)) == INV and st(moe(top=9)) == INV
    assert st(moe(hidden=48)) == UNS and st(moe(inter=40)) == UNS and st(moe(hidden=65568)) == UNS
    assert st(moe(n_experts=1025)) == UNS and st(moe(n_experts=64, top=33)) == UNS and st(moe(n_shared=63)) == UNS
    assert st(n=-1) == INV and st(n=1 << 31) == UNS and st(n=0) == 0 and st(n=0, x=0, ws=0) == 0
    for name in ("x", "y", "router", "up", "down"):
        assert st(**{name: 0}) == INV and st(**{name: 24}) == INV
    for name in ("experts", "w"):
        assert st(**{name: 0}) == INV and st(**{name: 18}) == INV
    assert st(bias=2) == INV and st(x_row=56) == INV and st(y_row=68) == UNS and st(x_row=(1 << 17) + 8) == UNS
    need = C.c_size_t()
    assert L.cs_moe_query(C.byref(moe()), 3, C.byref(need)) == 0 and need.value > 0
    assert st(ws_bytes=need.value - 1) == WS and str(need.value) in B.last_error() and st(ws=0) == INV and st(ws=8) == INV
    assert L.cs_moe_query(C.byref(moe()), 0, C.byref(need)) == 0 and need.value == 0
    assert L.cs_moe_query(C.byref(moe()), 3, None) == INV and L.cs_moe_query(C.byref(moe(top=0)), 3, C.byref(need)) == INV


def test_moe_workspace_stops_growing():
    sizes = []
    for n in (1, 2, 100, 4096, 5000, 1 << 30):
        need = C.c_size_t()
        assert B.lib().cs_moe_query(C.byref(moe()), n, C.byref(need)) == 0
        sizes.append(need.value)
    assert sizes == sorted(sizes) and sizes[3] == sizes[4] == sizes[5] < 1 << 30
    need = C.c_size_t()
    assert B.lib().cs_moe_query(C.byref(moe(hidden=65536, inter=65536, n_experts=64, n_shared=32, top=32)), 1 << 20, C.byref(need)) == 0


def test_the_binding_refuses_what_it_cannot_describe():
    import torch
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        B.cs_norm_residual(x, x, torch.ones(64))                   # not on the GPU
    with pytest.raises(ValueError, match="norm"):
        B.cs_norm_residual(x, x, torch.ones(64), norm="batch")
    with pytest.raises(ValueError):
        B.cs_weights_pack(x)
    with pytest.raises(TypeError):
        B.cs_weights_pack([[1.0]])
    with pytest.raises(ValueError):
        B.cs_weights_pack(x[0])
    p = B.PackedWeights(torch.zeros(1088, dtype=torch.uint8), "e2m1", 1, 16, 64)
    with pytest.raises(ValueError):
        B.cs_linear_packed(x, p)
    with pytest.raises(TypeError):
        B.cs_linear_packed(x, p, dtype=torch.float16)
    for weights in (x, None):
        with pytest.raises(TypeError):
            B.cs_linear_packed(x, weights)
        with pytest.raises(TypeError):
            B.cs_weights_read(weights)
        with pytest.raises(TypeError):
            B.cs_moe(x, x, weights, p, 2)
    with pytest.raises(ValueError):
        B.cs_moe(x, x, p, p, 2, score="max")


@pytest.mark.parametrize("kw", [dict(hidden=65536, inter=32, n_experts=32, n_shared=32, top=32), dict(hidden=65536, inter=65536, n_experts=32, n_shared=32, top=32),
                                dict(hidden=32, inter=65536, n_experts=1024, n_shared=32, top=32), dict(hidden=65536, inter=32, n_experts=1024, n_shared=63, top=1),
                                dict(hidden=7168, inter=2048, n_experts=256, n_shared=1, top=8), dict(hidden=2048, inter=768, n_experts=128, n_shared=0, top=8)])
def test_moe_workspace_is_bounded(kw):
    need = C.c_size_t()
    sizes = []
    for n in (1, 60, 1000, 4096, 1 << 20, (1 << 31) - 1):
        assert B.lib().cs_moe_query(C.byref(moe(**kw)), n, C.byref(need)) == 0
        sizes.append(need.value)
    assert sizes == sorted(sizes) and sizes[-1] == sizes[-2] == sizes[-3] <= 1 << 31
    # layers that fit take 4096 rows at once
    if kw["hidden"] <= 7168 and kw["inter"] <= 2048:
        assert B.lib().cs_moe_query(C.byref(moe(**kw)), 4095, C.byref(need)) == 0 and need.value < sizes[-1]


@pytest.mark.parametrize("args", [("e2m1", (1 << 32) + 48, 64), ("e2m1", 48, (1 << 32) + 64), ("bf16", -(1 << 32) + 48, 64), ("e2m1", 48, 64, (1 << 64) + 1),
                                  ("bf16", 1 << 31, 64)])
def test_sizes_that_do_not_fit_are_refused(args):
    with pytest.raises(ValueError, match="does not fit"):
        B.cs_weights_query(*args)


def test_overlapping_matrices_of_far_rows_are_refused():
    # (n - 1) w_row is past 64 bits
    c = weights(matrices=2, n=1 << 24)
    st = lambda row, matrix: B.lib().cs_weights_read(C.byref(c), 512, 256, row, matrix, B.CS_BF16, None)
    assert st(1 << 40, 1 << 50) == INV and "overlap" in B.last_error()
    assert st(1 << 39, 1 << 50) == INV and "overlap" in B.last_error()
