"""Norms around a block and packed weights on the GPU, against the CPU oracle."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as O
from paper_2603_12118_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(x, dtype="f32"):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV).to(TYPES[dtype])


def apart(x, pad):
    """The same rows, `pad` values further apart than they are long, with 7 between them."""
    wide = torch.full((x.shape[0], x.shape[1] + pad), 7.0, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def host(x):
    return None if x is None else x.double().cpu().numpy()


def within(got, want, bound, what):
    err = np.abs(host(got) - want)
    at = np.unravel_index(np.argmax(err - bound), err.shape) if err.size else None
    assert (err <= bound).all(), (what, at, err[at], bound[at])


def inputs(rows, width, dtype, residual, gate, post, kind, seed=0):
    rng = np.random.default_rng(seed)
    a = dict(x=dev(0.5 * rng.standard_normal((rows, width)) + 0.1, dtype), residual=dev(rng.standard_normal((rows, width)) * 3, residual),
             pre_gain=dev(1 + 0.1 * rng.standard_normal(width)))
    if kind == "layer":
        a["pre_bias"] = dev(0.1 * rng.standard_normal(width))
    if post:
        a["post_gain"] = dev(1 + 0.1 * rng.standard_normal(width))
        if kind == "layer":
            a["post_bias"] = dev(0.1 * rng.standard_normal(width))
    if gate:
        a["gate"] = dev(rng.standard_normal(width) if gate == "channel" else rng.standard_normal((rows, width)), dtype)
    return a


def check_norm(a, r, y, kind, dtype, residual, **kw):
    er, ey, dr, dy = O.norm_residual(*[host(a[k]) for k in ("x", "residual", "pre_gain")],
                                     **{k: host(a[k]) for k in ("pre_bias", "post_gain", "post_bias", "gate") if k in a}, kind=kind,
                                     r_type=residual, y_type=dtype, **kw)
    within(r, er, dr, "r")
    within(y, ey, dy, "y")


# widths on both sides of every number of lanes and pieces
@pytest.mark.parametrize("width", [8, 120, 504, 512, 520, 1024, 1032, 2048, 2056, 3584, 4096, 4104, 8192, 8200, 16384])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_widths(width, kind):
    a = inputs(5, width, "bf16", "f32", "row", True, kind, seed=width)
    r, y = B.cs_norm_residual(**a, residual_scale=0.7, block_scale=1.3, norm=kind)
    check_norm(a, r, y, kind, "bf16", "f32", residual_scale=np.float64(np.float32(0.7)), block_scale=np.float64(np.float32(1.3)))


@pytest.mark.parametrize("dtype,residual", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("kind,gate,post", [("rms", None, False), ("rms", "channel", True), ("layer", "row", False), ("layer", None, True), ("rms", "row", True)])
def test_types_gates_and_rows_apart(dtype, residual, kind, gate, post):
    rows, width = 131, 328
    a = inputs(rows, width, dtype, residual, gate, post, kind)
    a["x"], a["residual"] = apart(a["x"], 16), apart(a["residual"], 40)
    if gate == "row":
        a["gate"] = apart(a["gate"], 8)
    out, y = apart(torch.zeros_like(a["residual"]), 8), apart(torch.zeros_like(a["x"]), 24)
    got = B.cs_norm_residual(**a, norm=kind, eps=1e-3, r=out, y=y)
    assert got[0] is out and got[1] is y
    check_norm(a, out, y, kind, dtype, residual, eps=np.float64(np.float32(1e-3)))
    assert (out._base[:, width:] == 7).all() and (y._base[:, width:] == 7).all()


def test_in_place_and_the_same_bits():
    a = inputs(70, 3584, "bf16", "bf16", "channel", True, "rms")
    r, y = B.cs_norm_residual(**a)
    x, res = a["x"].clone(), a["residual"].clone()
    B.cs_norm_residual(**{**a, "x": x, "residual": res}, r=res, y=x)
    assert torch.equal(res, r) and torch.equal(x, y)
    one = [B.cs_norm_residual(**{**a, "x": a["x"][i:i + 1], "residual": a["residual"][i:i + 1]}) for i in (0, 69)]
    assert torch.equal(one[0][1][0], y[0]) and torch.equal(one[1][0][0], r[69])


def test_zero_rows_small_and_large_values():
    x = np.zeros((6, 64))
    x[1], x[2], x[3, 3] = 1e-20, 3.0, 1e4
    x[4] = np.linspace(-1, 1, 64) + 1000
    g = dev(np.ones(64))
    for kind in ("rms", "layer"):
        a = dict(x=dev(x), residual=dev(np.zeros((6, 64))), pre_gain=g, post_gain=g)
        r, y = B.cs_norm_residual(**a, norm=kind)
        check_norm(a, r, y, kind, "f32", "f32")
        assert not y[0].any() and torch.isfinite(y).all()
    r, y = B.cs_norm_residual(dev(x, "bf16"), dev(-x, "bf16"), g)          # what cancels is nothing
    assert not r.any() and not y.any()


def test_nan_and_infinity_stay_in_their_row():
    a = inputs(9, 512, "f32", "f32", None, True, "layer")
    want = B.cs_norm_residual(**a, norm="layer")
    a["x"][2, 77], a["residual"][6, 5] = float("nan"), float("inf")
    got = B.cs_norm_residual(**a, norm="layer")
    ok = [0, 1, 3, 4, 5, 7, 8]
    for w, g in zip(want, got):
        assert torch.equal(w[ok], g[ok])
    assert got[1][2].isnan().all() and got[1][6].isnan().any() and got[0][6, 5] == float("inf")


def test_more_rows_than_a_launch_takes():
    n = 4_194_303 + 70                                     # of 1024 threads: HIP's limit
    x, res, g = (torch.randn(n, 8, device=DEV, dtype=torch.bfloat16) for _ in range(2)), None, dev(1 + np.arange(8) / 8)
    x, res = x
    r, y = B.cs_norm_residual(x, res, g, post_gain=g)
    for at in (slice(0, 50), slice(4_194_250, 4_194_350), slice(n - 20, n)):
        check_norm(dict(x=x[at], residual=res[at], pre_gain=g, post_gain=g), r[at], y[at], "rms", "bf16", "bf16")
    assert torch.isfinite(y).all()


def test_on_another_stream_and_in_a_graph():
    a = inputs(37, 1024, "bf16", "f32", "row", True, "layer")
    side = torch.cuda.Stream()
    r, y = torch.empty_like(a["residual"]), torch.empty_like(a["x"])
    torch.cuda.synchronize()
    B.cs_norm_residual(**a, norm="layer", r=r, y=y, stream=side)
    side.synchronize()
    check_norm(a, r, y, "layer", "bf16", "f32")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cs_norm_residual(**a, norm="layer", r=r, y=y)
    for _ in range(3):
        a["x"].normal_()
        a["residual"].normal_()
        torch.cuda.synchronize()
        graph.replay()
        want = B.cs_norm_residual(**a, norm="layer")
        torch.cuda.synchronize()
        assert torch.equal(r, want[0]) and torch.equal(y, want[1])


def test_one_row_of_a_tensor_whose_rows_lie_anywhere():
    x, res = torch.randn(3, 68, device=DEV)[1:2, :64], torch.randn(3, 65, device=DEV)
    g = dev(np.ones(64))
    r, y = B.cs_norm_residual(x.bfloat16()[:, :64], res[:1, :64], g)          # 260 bytes apart
    assert r.shape == (1, 64) and torch.isfinite(y).all()
    with pytest.raises(B.CsError):
        B.cs_norm_residual(torch.randn(3, 64, device=DEV), res[:, :64], g)


def test_no_rows():
    g = dev(np.ones(64))
    r, y = B.cs_norm_residual(torch.zeros(0, 64, device=DEV), torch.zeros(0, 64, device=DEV), g)
    assert r.shape == y.shape == (0, 64)


# ---- weights
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("matrices,n,k", [(1, 1, 32), (1, 16, 128), (2, 17, 96), (3, 47, 160), (5, 33, 352)])
def test_weights_hold_what_the_format_says(matrices, n, k, dtype):
    rng = np.random.default_rng(n)
    w = dev(rng.standard_normal((matrices, n, k)) * 10.0 ** rng.integers(-4, 4, (matrices, n, 1)), dtype)
    wide = torch.full((matrices, n + 2, k + 8), 7.0, dtype=w.dtype, device=DEV)
    wide[:, :n, :k] = w
    for x in (w, wide[:, :n, :k]):
        flag = torch.zeros(1, dtype=torch.int32, device=DEV)
        p = B.cs_weights_pack(x, "e2m1", err_flag=flag)
        assert p.data.numel() == B.cs_weights_query("e2m1", n, k, matrices) and (p.matrices, p.n, p.k) == (matrices, n, k)
        for out in ("f32", "bf16"):
            assert np.array_equal(host(B.cs_weights_read(p, TYPES[out])), O.held(host(w), "e2m1"))
        b = B.cs_weights_pack(x, "bf16", err_flag=flag)
        assert torch.equal(B.cs_weights_read(b), w.bfloat16()) and flag.item() == 0
        # into a tensor with rows apart
        into = torch.full((matrices, n + 1, k + 16), 5.0, device=DEV)
        B.cs_weights_read(p, out=into[:, :n, :k])
        assert np.array_equal(host(into[:, :n, :k]), O.held(host(w), "e2m1")) and (into[:, n] == 5).all() and (into[:, :, k:] == 5).all()


def test_one_matrix_may_come_without_its_dimension():
    w = torch.randn(48, 64, device=DEV)
    assert torch.equal(B.cs_weights_pack(w).data, B.cs_weights_pack(w[None]).data)


@pytest.mark.parametrize("format", ["e2m1", "bf16"])
def test_matrices_of_one_row_that_lie_anywhere(format):
    # one row lies no distance from another: 67 values between rows that there are none of
    w = torch.randn(3, 67, device=DEV)[:1, :64]
    p = B.cs_weights_pack(w, format)
    assert torch.equal(p.data, B.cs_weights_pack(w.contiguous(), format).data)
    into = torch.full((1, 2, 67), 5.0, device=DEV)
    B.cs_weights_read(p, out=into[:, :1, :64])
    assert torch.equal(into[:, :1, :64], B.cs_weights_read(p, torch.float32)) and (into[:, 1] == 5).all() and (into[:, :, 64:] == 5).all()
    three = torch.randn(3, 1, 72, device=DEV)[:, :, :64]
    p = B.cs_weights_pack(three, format)
    assert torch.equal(p.data, B.cs_weights_pack(three.contiguous(), format).data)


def test_non_finite_weights_set_the_flag():
    w = torch.randn(2, 20, 64, device=DEV)
    w[1, 3, 4], w[0, 19, 63], w[0, 0, 0] = float("nan"), float("inf"), -float("inf")
    flag = torch.zeros(1, dtype=torch.int32, device=DEV)
    p = B.cs_weights_pack(w, err_flag=flag)
    assert flag.item() == 2 and np.array_equal(host(B.cs_weights_read(p, torch.float32)), O.held(host(w), "e2m1"))
    B.cs_weights_pack(w)                                   # without a flag


def test_weights_past_4_gib():
    # 4.3 GB of bf16 in 600 matrices
    w = torch.zeros(600, 1792, 2016, dtype=torch.bfloat16, device=DEV)
    w[599, 1791] = torch.randn(2016, device=DEV)
    p = B.cs_weights_pack(w, "bf16")
    assert p.data.numel() > 1 << 32
    q = B.cs_weights_read(p)
    assert torch.equal(q[599], w[599]) and not q[:599].any()
