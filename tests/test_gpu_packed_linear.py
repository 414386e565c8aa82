"""Products with packed weights on the GPU, against the CPU oracle."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as O
from paper_2603_12118_amd import binding as B
from tests.test_gpu_block import DEV, TYPES, apart, dev, host, within

pytestmark = pytest.mark.gpu


def make(rows, n, k, format, bias=True, seed=0):
    rng = np.random.default_rng(seed + 1000 * rows + n + k)
    x, w = dev(rng.standard_normal((rows, k)), "bf16"), dev(rng.standard_normal((n, k)) * k ** -0.5, "bf16")
    b = dev(rng.standard_normal(n)) if bias else None
    return x, w, b, B.cs_weights_pack(w, format)


def check(x, w, b, format, got, out):
    y, d = O.linear(host(x), O.held(host(w), format), host(b), out)
    within(got, y, d, (tuple(x.shape), tuple(w.shape), format, out))


# rows on both sides of every tile of rows, k of whole blocks and of one to three steps more, columns that end inside a tile and a workgroup
@pytest.mark.parametrize("format", ["e2m1", "bf16"])
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 32, 33, 48, 63, 65, 128, 129, 300])
def test_rows(rows, format):
    for n, k in ((48, 32), (1000, 96), (77, 128), (130, 1056), (512, 2208), (33, 1184)):
        x, w, b, p = make(rows, n, k, format)
        for out in ("bf16", "f32"):
            check(x, w, b, format, B.cs_linear_packed(x, p, bias=b, dtype=TYPES[out]), out)


# so many columns that a workgroup takes several tiles of them, with fewer waves along k than tiles
@pytest.mark.parametrize("format", ["e2m1", "bf16"])
@pytest.mark.parametrize("rows", [1, 3, 16, 30])
def test_many_columns(rows, format):
    for n, k in ((16397, 96), (4099, 64), (16384, 672), (4160, 352)):
        x, w, b, p = make(rows, n, k, format)
        for out in ("bf16", "f32"):
            check(x, w, b, format, B.cs_linear_packed(x, p, bias=b, dtype=TYPES[out]), out)


# two tiles of columns a workgroup, straight from memory (4 bits, 256 tiles and more, k that would be split): an odd number of tiles, columns that end
# inside the first and the second tile of a workgroup, k that ends inside a block; with one row, k beyond what LDS holds of it
@pytest.mark.parametrize("rows,n,k", [(rows, n, k) for rows in (2, 5, 16) for n in (4099, 4112, 4115, 4128) for k in (672, 1184)] +
                         [(1, n, 20512) for n in (4099, 4115)])
def test_two_tiles_of_columns_a_workgroup(rows, n, k):
    x, w, b, p = make(rows, n, k, "e2m1")
    for out in ("bf16", "f32"):
        y = apart(torch.zeros(rows, n, dtype=TYPES[out], device=DEV), 5)
        B.cs_linear_packed(x, p, bias=b, out=y)
        check(x, w, b, "e2m1", y, out)
        assert (y._base[:, n:] == 7).all()


@pytest.mark.parametrize("format", ["e2m1", "bf16"])
@pytest.mark.parametrize("rows", [1, 5, 20, 40, 100])
def test_long_rows_are_shared_out(rows, format):
    x, w, b, p = make(rows, 61, 12320, format, bias=False)
    check(x, w, b, format, B.cs_linear_packed(x, p, dtype=torch.float32), "f32")


# few rows on both sides of where they are staged
@pytest.mark.parametrize("format", ["e2m1", "bf16"])
@pytest.mark.parametrize("rows", [2, 6, 7, 15, 16])
def test_few_long_rows(rows, format):
    x, w, b, p = make(rows, 333, 16416, format)
    for out in ("bf16", "f32"):
        check(x, w, b, format, B.cs_linear_packed(x, p, bias=b, dtype=TYPES[out]), out)


# one row: both sides of what LDS holds of it
@pytest.mark.parametrize("format", ["e2m1", "bf16"])
@pytest.mark.parametrize("k", [20448, 20480, 20512])
def test_longest_rows_in_lds(k, format):
    x, w, b, p = make(1, 33, k, format)
    check(x, w, b, format, B.cs_linear_packed(x, p, bias=b, dtype=torch.float32), "f32")


@pytest.mark.parametrize("k", [96, 128, 416])
@pytest.mark.parametrize("rows", [1, 5, 20, 40, 60, 100])
def test_a_weight_that_is_no_number_leaves_the_other_columns(rows, k):
    x, w, b, p = make(rows, 83, k, "bf16")
    want = B.cs_linear_packed(x, p, bias=b)
    w[3, k - 1], w[82, 0], w[40, k // 2] = float("inf"), float("nan"), -float("inf")
    got = B.cs_linear_packed(x, B.cs_weights_pack(w, "bf16"), bias=b)
    ok = [j for j in range(83) if j not in (3, 40, 82)]
    assert torch.equal(got[:, ok], want[:, ok]) and not got[:, [3, 40, 82]].isfinite().any()


@pytest.mark.parametrize("rows", [3, 30, 90])
def test_rows_apart_and_results_apart(rows):
    for n, gap in ((96, 8), (96, 2), (96, 1), (95, 3)):
        x, w, b, p = make(rows, n, 288, "e2m1")
        x = apart(x, 16)
        for out in ("bf16", "f32"):
            y = apart(torch.zeros(rows, n, dtype=TYPES[out], device=DEV), gap)
            assert B.cs_linear_packed(x, p, bias=b, out=y) is y
            check(x, w, b, "e2m1", y, out)
            assert (y._base[:, n:] == 7).all()


@pytest.mark.parametrize("format", ["e2m1", "bf16"])
@pytest.mark.parametrize("rows", [9, 50, 140])
def test_a_row_with_a_nan_leaves_the_others(rows, format):
    x, w, b, p = make(rows, 200, 416, format)
    want = B.cs_linear_packed(x, p, bias=b)
    x[rows - 2, 415], x[0, 0] = float("nan"), float("inf")
    got = B.cs_linear_packed(x, p, bias=b)
    ok = [i for i in range(rows) if i not in (0, rows - 2)]
    assert torch.equal(got[ok], want[ok]) and got[rows - 2].isnan().all() and not got[0].isfinite().any()


@pytest.mark.parametrize("rows", [8, 60, 200])
def test_workspace_stream_and_graph(rows):
    x, w, b, p = make(rows, 300, 4096, "e2m1")
    want = B.cs_linear_packed(x, p, bias=b)
    work = torch.full((1 << 26,), 255, dtype=torch.uint8, device=DEV)          # NaNs: what it held is not read
    assert torch.equal(B.cs_linear_packed(x, p, bias=b, workspace=work), want)
    assert torch.equal(B.cs_linear_packed(x, p, bias=b, workspace=work[:16]), want)
    side, y = torch.cuda.Stream(), torch.empty_like(want)
    torch.cuda.synchronize()
    B.cs_linear_packed(x, p, bias=b, out=y, workspace=work, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cs_linear_packed(x, p, bias=b, out=y)
    for i in range(3):
        x.copy_(torch.randn(rows, 4096, device=DEV))
        torch.cuda.synchronize()
        graph.replay()
        want = B.cs_linear_packed(x, p, bias=b)
        torch.cuda.synchronize()
        assert torch.equal(y, want), i


def test_no_rows_and_many():
    x, w, b, p = make(5000, 40, 64, "e2m1")
    check(x, w, b, "e2m1", B.cs_linear_packed(x, p, bias=b, dtype=torch.float32), "f32")
    assert B.cs_linear_packed(x[:0], p).shape == (0, 40)
