"""More rows than the grid of one launch has workgroups for (2^32 - 1 threads): as if they were given in parts."""
import pytest
import torch

from paper_2603_12118_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MOST = (2 ** 32 - 1) // 256


def room(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of device memory")


def test_queries_normed_and_rotated():
    room(24)
    T = 4 * MOST + 1003
    gen = torch.Generator(DEV).manual_seed(0)
    q = torch.randn(T, 1, 16, generator=gen, device=DEV, dtype=torch.bfloat16)
    cs = torch.randn(7, 8, 2, generator=gen, device=DEV)
    pos = torch.randint(0, 7, (T, 2), generator=gen, device=DEV, dtype=torch.int32)
    gain = torch.randn(16, generator=gen, device=DEV)
    flag = torch.zeros(1, dtype=torch.int32, device=DEV)
    for K in (0, 1):
        k = torch.randn(T, K, 16, generator=gen, device=DEV, dtype=torch.bfloat16)
        qo, ko = B.cs_qk_norm_rope(q, k, cs, pos, (3, 5), gain, gain, err_flag=flag)
        for a, b in ((0, 4 * MOST - 9), (4 * MOST - 9, T)):
            want = B.cs_qk_norm_rope(q[a:b], k[a:b], cs, pos[a:b], (3, 5), gain, gain, err_flag=flag)
            assert torch.equal(qo[a:b], want[0]) and torch.equal(ko[a:b], want[1])
    assert flag.item() == 0 and not torch.equal(qo, q)


def test_rows_into_the_cache_and_out_of_it():
    room(160)
    T, P = 16 * MOST + 777, 64
    edges = [(0, 50), (16 * MOST - 20, 16 * MOST + 30), (T - 40, T)]
    gen = torch.Generator(DEV).manual_seed(1)
    slots = torch.full((T,), -1, dtype=torch.int64, device=DEV)
    k, v = (torch.empty(T, 1, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    at = 0
    for a, b in edges:
        slots[a:b] = torch.arange(at, at + b - a, device=DEV)
        k[a:b], v[a:b] = (torch.randn(b - a, 1, 128, generator=gen, device=DEV, dtype=torch.bfloat16) for _ in range(2))
        at += b - a
    pool, parts = (torch.zeros(3, P * 136, dtype=torch.uint8, device=DEV) for _ in range(2))
    flag = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.cs_cache_write(pool, k, v, slots, P, err_flag=flag)
    for a, b in edges:
        B.cs_cache_write(parts, k[a:b], v[a:b], slots[a:b], P, err_flag=flag)
    assert pool.any() and torch.equal(pool, parts)
    wanted = [B.cs_cache_read(pool, slots[a:b], 1, 128, P) for a, b in edges]
    B.cs_cache_read(pool, slots, 1, 128, P, k=k, v=v, err_flag=flag)
    for (a, b), (wk, wv) in zip(edges, wanted):
        assert torch.equal(k[a:b], wk) and torch.equal(v[a:b], wv)
    assert not k[50:10 ** 6].any() and not v[T - 700:T - 40].any() and flag.item() == 0
