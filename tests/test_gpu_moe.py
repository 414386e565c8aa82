"""The mixture-of-experts layer on the GPU, against the CPU oracle."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import block_oracle as O
from paper_2603_12118_amd import binding as B
from tests.test_gpu_block import DEV, apart, dev, host, within

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, hidden, inter, experts, shared, format, seed=0):
        rng = np.random.default_rng(seed + hidden + experts)
        self.router = dev(rng.standard_normal((experts, hidden)) * hidden ** -0.5, "bf16")
        up, down = (dev(rng.standard_normal(s) * s[-1] ** -0.5, "bf16") for s in ((experts + shared, 2 * inter, hidden), (experts + shared, hidden, inter)))
        self.up, self.down = B.cs_weights_pack(up, format), B.cs_weights_pack(down, format)
        self.held = O.held(host(up), format), O.held(host(down), format)
        self.bias = dev(0.05 * rng.standard_normal(experts))
        self.rng, self.hidden = rng, hidden

    def rows(self, n):
        return dev(self.rng.standard_normal((n, self.hidden)), "bf16")

    def check(self, x, top, got=None, **kw):
        if got is None:
            got = B.cs_moe(x, self.router, self.up, self.down, top, **kw)
        okw = {k: host(v) if k == "choice_bias" else v.cpu().numpy() != 0 if k == "live" else v for k, v in kw.items() if k in (
            "score", "renormalise", "scale", "choice_bias", "live") and v is not None}
        if "scale" in okw:
            okw["scale"] = float(np.float32(okw["scale"]))
        y, experts, weights, d = O.moe(host(x), host(self.router), *self.held, top, **okw)
        assert np.array_equal(got[1].cpu().numpy(), experts)
        within(got[2], weights, 2.0 ** -24 * np.abs(weights) * 1.001, "weights")
        within(got[0], y, d, "y")
        return got


@pytest.mark.parametrize("format", ["e2m1", "bf16"])
@pytest.mark.parametrize("hidden,inter,experts,top,shared", [(64, 32, 4, 2, 0), (96, 352, 24, 3, 0), (512, 96, 200, 10, 0), (1056, 64, 5, 5, 2),
                                                             (256, 160, 3, 1, 1), (128, 32, 300, 32, 3), (64, 96, 1, 1, 0)])
def test_layers(hidden, inter, experts, top, shared, format):
    layer = Layer(hidden, inter, experts, shared, format)
    for rows in (1, 2, 3, 7, 33):
        layer.check(layer.rows(rows), top)


# as many experts as there may be, most of them without a row
@pytest.mark.parametrize("rows", [1, 2, 16, 40, 90])
def test_many_experts(rows):
    layer = Layer(64, 32, 1000, 24, "e2m1")
    layer.check(layer.rows(rows), 32)
    layer.check(layer.rows(rows), 1, choice_bias=layer.bias)


# the widest layers that the calls take
@pytest.mark.parametrize("hidden,inter", [(65536, 32), (64, 65536)])
@pytest.mark.parametrize("rows", [1, 3, 70])
def test_widest_layers(hidden, inter, rows):
    layer = Layer(hidden, inter, 2, 1, "e2m1")
    layer.check(layer.rows(rows), 1)


# second products over rows that LDS holds whole, and longer ones
@pytest.mark.parametrize("format", ["e2m1", "bf16"])
@pytest.mark.parametrize("inter", [1120, 1152, 1184])
def test_long_second_products(inter, format):
    layer = Layer(160, inter, 5, 1, format)
    for rows in (3, 75, 200):
        layer.check(layer.rows(rows), 3)


# experts with every number of tiles of rows, and more rows than a workgroup takes at once
@pytest.mark.parametrize("rows", [1, 5, 16, 17, 40, 64, 65, 100, 190, 515])
def test_rows(rows):
    layer = Layer(128, 64, 6, 1, "e2m1")
    layer.check(layer.rows(rows), 2)


# few rows on both sides of where second products and the sum get launches of their own, one of them idle
@pytest.mark.parametrize("format", ["e2m1", "bf16"])
@pytest.mark.parametrize("rows", [2, 8, 9, 16])
def test_few_rows_of_many_experts(rows, format):
    layer = Layer(96, 352, 64, 1, format)
    layer.check(layer.rows(rows), 6)
    layer.check(layer.rows(rows), 6, live=torch.arange(rows, device=DEV) != rows - 2)


@pytest.mark.parametrize("format", ["e2m1", "bf16"])
def test_all_rows_take_the_same_experts(format):
    # 700 rows for two of 32 experts, the average being 44
    layer = Layer(64, 32, 32, 0, format)
    x = layer.rows(700)
    layer.check(x, 2, score="sigmoid", choice_bias=dev(np.where(np.isin(np.arange(32), (7, 30)), 10.0, 0.0)))


@pytest.mark.parametrize("rows", [1, 2, 30, 200])
@pytest.mark.parametrize("kw", [dict(score="sigmoid", scale=2.5), dict(score="sigmoid", choice_bias=True), dict(choice_bias=True, renormalise=False),
                                dict(renormalise=False, scale=-0.3)])
def test_scores(rows, kw):
    layer = Layer(160, 32, 40, 1, "e2m1")
    kw = dict(kw)
    if kw.get("choice_bias"):
        kw["choice_bias"] = layer.bias
    layer.check(layer.rows(rows), 6, **kw)


@pytest.mark.parametrize("rows", [1, 2, 20, 150])
def test_idle_rows(rows):
    layer = Layer(128, 64, 9, 2, "e2m1")
    clean = layer.rows(rows)
    for live in (torch.arange(rows, device=DEV) % 3 != 1, torch.zeros(rows, dtype=torch.bool, device=DEV), torch.ones(rows, dtype=torch.uint8, device=DEV)):
        x = clean.clone()
        x[live == 0] = float("nan")
        y, experts, weights = B.cs_moe(x, layer.router, layer.up, layer.down, 3, live=live)
        dead = live == 0
        assert not y[dead].any() and (experts[dead] == -1).all() and not weights[dead].any()
        if live.any():
            layer.check(x[live != 0], 3, got=tuple(v[live != 0] for v in (y, experts, weights)))
            alone = B.cs_moe(x[live != 0], layer.router, layer.up, layer.down, 3)
            assert torch.equal(alone[1], experts[live != 0])


@pytest.mark.parametrize("rows", [1, 4, 50])
def test_equal_scores_take_the_lowest_numbers(rows):
    layer = Layer(64, 32, 70, 0, "e2m1")
    layer.router[10:] = layer.router[:60].clone()            # expert e + 10 scores as e does
    got = layer.check(layer.rows(rows), 8)
    layer.router.zero_()
    got = layer.check(layer.rows(rows), 8)
    assert (got[1] == torch.arange(8, device=DEV)).all()


@pytest.mark.parametrize("rows", [1, 2, 40])
def test_nan_and_infinity_stay_in_their_row(rows):
    layer = Layer(96, 64, 12, 1, "bf16")
    x = layer.rows(rows + 2)
    want = B.cs_moe(x[1:-1].contiguous(), layer.router, layer.up, layer.down, 3)
    x[0, 5], x[-1, 90] = float("nan"), float("inf")
    got = B.cs_moe(x, layer.router, layer.up, layer.down, 3)
    assert torch.equal(got[1][1:-1], want[1]) and torch.equal(got[2][1:-1], want[2])
    layer.check(x[1:-1], 3, got=tuple(g[1:-1] for g in got))
    assert got[0][0].isnan().all() and ((got[1] >= 0) & (got[1] < 12)).all()
    one = B.cs_moe(x[:1], layer.router, layer.up, layer.down, 3)
    assert one[0].isnan().all() and (one[1][0] == torch.arange(3, device=DEV)).all()


def test_the_same_bits_every_time_and_for_every_batch_of_a_kind():
    layer = Layer(512, 96, 16, 1, "e2m1")
    x = layer.rows(200)
    first = B.cs_moe(x, layer.router, layer.up, layer.down, 4)
    for _ in range(5):
        again = B.cs_moe(x, layer.router, layer.up, layer.down, 4)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_rows_apart_workspace_stream_and_graph():
    layer = Layer(256, 96, 20, 1, "e2m1")
    for rows in (1, 6, 100):
        x = apart(layer.rows(rows), 40)
        args = (layer.router, layer.up, layer.down, 4)
        want = B.cs_moe(x, *args)
        work = torch.full((1 << 25,), 255, dtype=torch.uint8, device=DEV)
        y = apart(torch.zeros(rows, 256, dtype=torch.bfloat16, device=DEV), 8)
        experts, weights = torch.empty(rows, 4, dtype=torch.int32, device=DEV), torch.empty(rows, 4, device=DEV)
        out = dict(y=y, experts=experts, weights=weights)
        got = B.cs_moe(x, *args, workspace=work, **out)
        assert got[0] is y and got[1] is experts and got[2] is weights
        assert all(torch.equal(a, b) for a, b in zip(want, got)) and (y._base[:, 256:] == 7).all()
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        y.zero_()
        torch.cuda.synchronize()
        B.cs_moe(x, *args, workspace=work, stream=side, **out)
        side.synchronize()
        assert torch.equal(y, want[0])
        graph = torch.cuda.CUDAGraph()
        live = torch.ones(rows, dtype=torch.bool, device=DEV)
        with torch.cuda.graph(graph):
            B.cs_moe(x, *args, live=live, **out)
        for i in range(4):
            x.copy_(torch.randn(rows, 256, device=DEV))
            if rows > 1:
                live.copy_(torch.rand(rows, device=DEV) < 0.8)
            torch.cuda.synchronize()
            graph.replay()
            want = B.cs_moe(x, *args, live=live)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, (y, experts, weights))), (rows, i)


def test_more_rows_than_go_together():
    layer = Layer(64, 32, 8, 0, "e2m1")
    x = layer.rows(4096 + 37)
    live = torch.rand(len(x), device=DEV) < 0.9
    got = B.cs_moe(x, layer.router, layer.up, layer.down, 2, live=live)
    layer.check(x[4000:], 2, got=tuple(g[4000:] for g in got), live=live[4000:])
    tail = B.cs_moe(x[4096:], layer.router, layer.up, layer.down, 2, live=live[4096:])
    assert torch.equal(tail[1], got[1][4096:])
    # behind the first 4096 a few, one, or none
    for n in (4096 + 9, 4097, 4096):
        got = B.cs_moe(x[:n], layer.router, layer.up, layer.down, 2)
        layer.check(x[4060:n], 2, got=tuple(g[4060:] for g in got))


def test_no_rows():
    layer = Layer(64, 32, 8, 0, "e2m1")
    y, experts, weights = B.cs_moe(layer.rows(0), layer.router, layer.up, layer.down, 2)
    assert y.shape == (0, 64) and experts.shape == weights.shape == (0, 2)


def test_more_rows_than_the_workspace_holds():
    # a layer so wide that its workspace's bound and not the number of rows ends a group
    layer = Layer(65536, 32, 2, 14, "bf16")
    c, need = B.cs_moe_config(C.sizeof(B.cs_moe_config), B.CS_WEIGHTS_BF16, 65536, 32, 2, 14, 2, B.CS_SCORE_SOFTMAX, 1, 1.0), C.c_size_t()

    def size(n):
        assert B.lib().cs_moe_query(C.byref(c), n, C.byref(need)) == 0
        return need.value
    group = next(n for n in range(1, 4096) if size(n) == size(n + 1))
    assert 64 < group < 4000 and size(group - 1) < size(group) == size(1 << 20) <= 1 << 31
    x = layer.rows(group + 21)
    live = torch.arange(len(x), device=DEV) % 7 != 3
    work = torch.full((size(group),), 255, dtype=torch.uint8, device=DEV)          # NaNs, and no byte more than is asked for
    for n in (len(x), group + 1, group):
        got = B.cs_moe(x[:n], layer.router, layer.up, layer.down, 2, live=live[:n], workspace=work)
        assert got[0].isfinite().all() and not got[0][~live[:n]].any() and got[0][live[:n]].any(-1).all()
        for at in (slice(0, 3), slice(group - 3, min(n, group + 21))):
            layer.check(x[:n][at], 2, got=tuple(g[at] for g in got), live=live[:n][at])


# A row's bits do not depend on the rows beside it, while the call takes the same launches: rows in another order, and fewer of them, so that lists
# end inside 16, 32, 48 and 64 rows.  Second products whole in LDS, through stages, and few rows straight from memory.
@pytest.mark.parametrize("format", ["e2m1", "bf16"])
@pytest.mark.parametrize("hidden,inter,experts,top,shared,counts", [(512, 96, 16, 4, 1, (200, 193, 177, 150, 131, 64)), (160, 1184, 5, 2, 1, (190, 170, 143, 100, 70)),
                                                                    (96, 352, 200, 10, 0, (110, 97, 83, 64)), (96, 352, 64, 3, 1, (60, 41, 17))])
def test_rows_have_the_same_bits_beside_other_rows(hidden, inter, experts, top, shared, counts, format):
    layer = Layer(hidden, inter, experts, shared, format)
    x = layer.rows(counts[0])
    first = B.cs_moe(x, layer.router, layer.up, layer.down, top)
    layer.check(x, top, got=first)
    for n in counts:
        for seed in range(3):
            rows = torch.from_numpy(np.random.default_rng(seed + n).permutation(counts[0])[:n]).to(DEV)
            got = B.cs_moe(x[rows], layer.router, layer.up, layer.down, top)
            for a, b, name in zip(first, got, ("y", "experts", "weights")):
                assert torch.equal(a[rows], b), (n, seed, name)
