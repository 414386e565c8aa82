"""The 4-bit cache on the GPU against the CPU oracle: every byte written, every value read."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2603_12118_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev_rows(x, dtype, pad=0):
    """[T, heads, D] on the GPU, rows `pad` heads further apart than they are long."""
    T, H, D = x.shape
    wide = torch.full((T, H + pad, D), 7.0, dtype=TYPES[dtype], device=DEV)
    wide[:, :H] = torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    return wide[:, :H]


def as_held(x, dtype):
    """What the rows are after their storage type."""
    return x.to(TYPES[dtype]).double().cpu().numpy() if isinstance(x, torch.Tensor) else x


def fresh(heads, dim, page, pages, seed=0):
    return np.random.default_rng(seed).integers(0, 256, (pages, heads * page * (dim + dim // 16)), dtype=np.uint8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,dim,page", [(1, 1, 128, 32), (3, 4, 128, 64), (17, 2, 64, 32), (95, 5, 128, 96), (131, 3, 64, 160),
                                                 (64, 1, 64, 1024)])
def test_every_byte_written(rows, heads, dim, page, dtype):
    rng = np.random.default_rng(rows)
    pages = -(-rows // page) + 2
    pool = fresh(heads, dim, page, pages)
    slots = rng.permutation(pages * page)[:rows].astype(np.int64)
    slots[rows // 2] = -1
    k, v = (dev_rows(rng.standard_normal((rows, heads, dim)) * 10.0 ** rng.integers(-4, 4, (rows, heads, 1)), dtype, pad=p) for p in (0, 3))
    dpool, flag = torch.from_numpy(pool).to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    B.cs_cache_write(dpool, k, v, torch.from_numpy(slots).to(DEV), page, err_flag=flag)
    want = O.write(pool, as_held(k, dtype), as_held(v, dtype), slots, page)
    assert np.array_equal(dpool.cpu().numpy(), want) and flag.item() == 0
    # and back, into rows that lie apart
    for out in ("bf16", "f32"):
        rk, rv = dev_rows(np.zeros((rows, heads, dim)), out, pad=1), dev_rows(np.zeros((rows, heads, dim)), out)
        B.cs_cache_read(dpool, torch.from_numpy(slots).to(DEV), heads, dim, page, dtype=TYPES[out], k=rk, v=rv, err_flag=flag)
        ek, ev = O.read(want, slots, heads, dim, page)
        assert np.array_equal(rk.double().cpu().numpy(), ek) and np.array_equal(rv.double().cpu().numpy(), ev) and flag.item() == 0
        assert not rk[rows // 2].any() and (rk._base[:, heads] == 7).all()


def test_consecutive_rows_of_a_prompt():
    # pages filled end to end, one of them ending inside a workgroup's rows
    rng = np.random.default_rng(5)
    pool = fresh(2, 128, 32, 6)
    order = np.array([4, 1, 5, 0, 3])
    t = np.arange(150)
    slots = order[t // 32] * 32 + t % 32
    k, v = (dev_rows(rng.standard_normal((150, 2, 128)), "bf16") for _ in range(2))
    dpool = torch.from_numpy(pool).to(DEV)
    B.cs_cache_write(dpool, k, v, torch.from_numpy(slots).to(DEV), 32)
    assert np.array_equal(dpool.cpu().numpy(), O.write(pool, as_held(k, "bf16"), as_held(v, "bf16"), slots, 32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties_small_large_and_non_finite_values(dtype):
    x = np.zeros((10, 1, 64))
    x[0, 0, :8] = [6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5]
    x[0, 0, 8:16] = [-.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, 0.0]
    x[1, 0, :3] = [7.0, 6.97, 5.0]                       # the scale moves up
    x[1, 0, 32:36] = [6.96875, 5.0, -5.0, 1e-9]          # and does not: bf16 below 7
    x[2, 0, :4] = [1e-38, 3e-39, -1e-38, 1e-30]          # below the smallest scale
    x[2, 0, 32:34] = [2.0 ** -126, 2.0 ** -124]
    x[3, 0, :3] = [3.3e38, -2.9e38, 1e38]
    x[4, 0, 5], x[4, 0, 40] = np.inf, -np.inf
    x[5, 0, 3], x[5, 0, 4], x[5, 0, 60] = np.nan, 2.0, -np.nan
    x[6] = -0.0
    x[7, 0, ::2], x[7, 0, 1] = np.nan, np.inf
    x[8, 0] = np.linspace(-7, 7, 64)
    x[9, 0] = 2.0 ** np.arange(-32, 32)
    k = dev_rows(x, dtype)
    v = dev_rows(x[::-1].copy(), dtype)
    pool, slots = fresh(1, 64, 32, 1), np.arange(3, 13)
    dpool, flag = torch.from_numpy(pool).to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    B.cs_cache_write(dpool, k, v, torch.from_numpy(slots).to(DEV), 32, err_flag=flag)
    want = O.write(pool, as_held(k, dtype), as_held(v, dtype), slots, 32)
    assert flag.item() == 2
    gk, gv = B.cs_cache_read(dpool, torch.from_numpy(slots).to(DEV), 1, 64, 32, dtype=torch.float32)
    ek, ev = O.read(want, slots, 1, 64, 32)
    assert np.array_equal(gk.double().cpu().numpy(), ek) and np.array_equal(gv.double().cpu().numpy(), ev)
    assert np.isfinite(ek).all() and np.array_equal(ek, O.held(as_held(k, dtype)))


def test_finite_rows_leave_the_flag_and_bad_slots_are_left_out():
    rng = np.random.default_rng(6)
    pool = fresh(2, 64, 32, 2)
    slots = np.array([0, 64, -2, 63, 1 << 40, -(1 << 62), -1], np.int64)
    k, v = (dev_rows(rng.standard_normal((7, 2, 64)), "f32") for _ in range(2))
    dpool, flag = torch.from_numpy(pool).to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    dslots = torch.from_numpy(slots).to(DEV)
    B.cs_cache_write(dpool, k, v, dslots, 32, err_flag=flag)
    want = O.write(pool, as_held(k, "f32"), as_held(v, "f32"), slots, 32)
    assert np.array_equal(dpool.cpu().numpy(), want) and flag.item() == 1
    flag.zero_()
    gk, gv = B.cs_cache_read(dpool, dslots, 2, 64, 32, dtype=torch.float32, err_flag=flag)
    ek, ev = O.read(want, slots, 2, 64, 32)
    assert np.array_equal(gk.double().cpu().numpy(), ek) and np.array_equal(gv.double().cpu().numpy(), ev) and flag.item() == 1
    flag.zero_()
    B.cs_cache_read(dpool, dslots[[0, 3, 6]], 2, 64, 32, err_flag=flag)
    B.cs_cache_write(dpool, k[[0, 3, 6]], v[[0, 3, 6]], dslots[[0, 3, 6]], 32, err_flag=flag)
    B.cs_cache_write(dpool, k, v, dslots, 32)                          # without a flag
    assert flag.item() == 0
    B.cs_cache_write(dpool, k[:0], v[:0], dslots[:0], 32)              # no rows
    assert B.cs_cache_read(dpool, dslots[:0], 2, 64, 32)[0].shape == (0, 2, 64)


def test_a_pool_past_4_gib():
    # 32 000 pages of 8 heads x 128 tokens: 4.46 GB
    heads, page, pages = 8, 128, 32000
    pool = torch.zeros(pages, heads * page * 136, dtype=torch.uint8, device=DEV)
    assert pool.numel() > 1 << 32
    rng = np.random.default_rng(8)
    k, v = (dev_rows(rng.standard_normal((4, heads, 128)), "bf16") for _ in range(2))
    slots = torch.tensor([pages * page - 1, (pages - 1) * page, 31000 * page + 77, 5], device=DEV)
    B.cs_cache_write(pool, k, v, slots, page)
    gk, gv = B.cs_cache_read(pool, slots, heads, 128, page, dtype=torch.float32)
    assert np.array_equal(gk.double().cpu().numpy(), O.held(as_held(k, "bf16")))
    assert np.array_equal(gv.double().cpu().numpy(), O.held(as_held(v, "bf16")))
    assert int((pool[6:31000] != 0).sum()) == 0


def test_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(9)
    side = torch.cuda.Stream()
    pool = torch.zeros(4, 2 * 32 * 136, dtype=torch.uint8, device=DEV)
    k, v = (dev_rows(rng.standard_normal((20, 2, 128)), "bf16") for _ in range(2))
    slots = torch.arange(20, device=DEV) * 5
    torch.cuda.synchronize()
    B.cs_cache_write(pool, k, v, slots, 32, stream=side)
    gk, gv = B.cs_cache_read(pool, slots, 2, 128, 32, dtype=torch.float32, stream=side)
    side.synchronize()
    assert np.array_equal(gk.double().cpu().numpy(), O.held(as_held(k, "bf16")))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cs_cache_write(pool, k, v, slots, 32)
        B.cs_cache_read(pool, slots, 2, 128, 32, k=gk, v=gv, dtype=torch.float32)
    for i in range(4):                                                 # new rows and slots between the replays
        k.copy_(torch.randn(20, 2, 128, device=DEV))
        slots.copy_(torch.randperm(128, device=DEV)[:20])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(gk.double().cpu().numpy(), O.held(as_held(k, "bf16"))), i
        assert np.array_equal(gv.double().cpu().numpy(), O.held(as_held(v, "bf16"))), i
