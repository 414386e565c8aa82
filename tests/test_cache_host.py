"""The LLM task's attention calls without a GPU: the CPU oracle against brute force, and what the calls refuse before
anything is enqueued."""
import ctypes as C

import numpy as np
import pytest

from oracle import cache_oracle as O
from paper_2603_12118_amd import binding as B


# ---- the oracle
def test_quantise_takes_the_nearest_level_and_even_codes_on_ties():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(64 * 32) * 10.0 ** rng.integers(-6, 6, 64).repeat(32),
                        np.array([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5] * 4),            # every tie, scale 1
                        np.array([7 - 1e-9, 5.0, -0.25, -5] * 8), np.array([7.0, 5, 3, 1] * 8), np.zeros(32)]).reshape(-1, 32)
    codes, scales = O.quantise(x)
    got = O.values(codes, scales)
    for row, c, s, v in zip(x, codes, scales, got):
        top = np.abs(row).max()
        if not top:
            assert s[0] == 2 and not v.any()
            continue
        unit = 2.0 ** (int(s[0]) - 127)
        assert 3.5 * unit <= top < 7 * unit                      # the largest rounds to 4 units or more, and none is clipped by more than one
        for xi, ci, vi in zip(row, c, v):
            assert abs(vi - xi) == min(abs(np.sign(xi) * l * unit - xi) for l in O.LEVELS)
            assert (abs(abs(xi) / unit % 0.5 - 0.25) > 1e-12 or ci % 2 == 0) or abs(xi) >= 2 * unit
    ties = O.quantise(np.array([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5] * 4).reshape(1, 32))
    assert ties[1][0, 0] == 127 and list(ties[0][0, :8]) == [7, 0, 2, 2, 4, 4, 6, 6]
    assert list(O.held(np.array([[np.nan, np.inf, -np.inf, 0] + [0] * 28]))[0, :3]) == [0.0, 6 * 2.0 ** 125, -6 * 2.0 ** 125]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [32, 96])
def test_every_byte_of_a_block_belongs_to_one_place(dim, page):
    at = np.concatenate([np.concatenate(O.code_addresses(o, page, dim)) for o in range(page)])
    assert sorted(at) == list(range(page * (dim + dim // 16)))
    assert B.cs_cache_query(3, dim, page, 5) == (3 * len(at), 15 * len(at))


def test_written_rows_read_back():
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((2, 7, 2, 64))
    pool = rng.integers(0, 256, (3, 2 * 32 * 68), dtype=np.uint8)
    slots = np.array([5, 90, -1, 33, 0, 96, 40])                 # 96: beyond the pool
    new = O.write(pool, k, v, slots, 32)
    rk, rv = O.read(new, slots, 2, 64, 32)
    ok = [0, 1, 3, 4, 6]
    assert np.array_equal(rk[ok], O.held(k)[ok]) and np.array_equal(rv[ok], O.held(v)[ok])
    assert not rk[[2, 5]].any() and (new != pool).sum() <= 5 * 2 * 2 * (32 + 2)


def test_attention_of_the_oracle_against_a_direct_sum():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((5, 4, 8)), rng.standard_normal((6, 2, 8)), rng.standard_normal((6, 2, 8))
    out, weight = O.attention(q, [k, k[:2]], [v, v[:2]], [2, 3], 0.3)
    for t, h, n, kk, vv in ((0, 0, 5, k, v), (1, 3, 6, k, v), (3, 1, 1, k[:2], v[:2]), (4, 2, 2, k[:2], v[:2])):
        e = [np.exp(0.3 * float(q[t, h] @ kk[j, h // 2])) for j in range(n)]
        assert np.allclose(out[t, h], sum(w * vv[j, h // 2] for j, w in enumerate(e)) / sum(e), rtol=1e-13)
    assert not out[2].any() and not weight[2].any()              # query 0 of a sequence with fewer keys than queries
    full, _ = O.attention(q, [k, k[:2]], [v, v[:2]], [2, 3], 0.3, causal=False)
    assert full[2].any() and np.allclose(full[1], out[1])


def test_axes_of_rotary_pairs():
    assert list(O.axis_of_pairs((2, 1, 3), False)) == [0, 0, 1, 2, 2, 2]
    assert list(O.axis_of_pairs((4, 2, 2), True)) == [0, 1, 2, 0, 1, 2, 0, 0]
    x = np.random.default_rng(3).standard_normal((3, 2, 24))
    ang = np.random.default_rng(4).standard_normal((9, 8))
    cs = np.stack((np.cos(ang), np.sin(ang)), -1)
    pos = np.array([[0, 3, 8], [1, 1, 1], [7, 2, 5]])
    y = O.norm_rope(x, cs, pos, (4, 2, 2), interleaved=True)
    z = x[..., :8] + 1j * x[..., 8:16]
    for j, a in enumerate([0, 1, 2, 0, 1, 2, 0, 0]):
        r = z[:, :, j] * np.exp(1j * ang[pos[:, a], j])[:, None]
        assert np.allclose(y[..., j] + 1j * y[..., 8 + j], r)
    assert np.array_equal(y[..., 16:], x[..., 16:])
    g = np.arange(1, 25.0)
    assert np.allclose(O.norm_rope(x, cs, 0 * pos, (4, 2, 2), gain=g, eps=0.5)[..., 20], x[..., 20] * 21 / np.sqrt((x ** 2).mean(-1) + .5))


# ---- refusals: pointers here are plain numbers, nothing is enqueued
INV, WS, UNS = B.CS_ERR_INVALID_ARG, B.CS_ERR_WORKSPACE, B.CS_ERR_UNSUPPORTED


def cache(**kw):
    d = dict(n_kv_heads=2, head_dim=128, page_tokens=32, n_pages=4) | kw
    return B.cs_cache_config(d.pop("struct_size", C.sizeof(B.cs_cache_config)), **d)


def write_status(c, k=64, k_row=256, v=128, v_row=256, dtype=None, slots=16, n=4, pool=256, err=None, call="cs_cache_write"):
    f, dt = getattr(B.lib(), call), B.CS_BF16 if dtype is None else dtype
    if call == "cs_cache_write":
        return f(C.byref(c) if c else None, pool, k, k_row, v, v_row, dt, slots, n, err, None)
    return f(C.byref(c) if c else None, pool, slots, n, k, k_row, v, v_row, dt, err, None)


@pytest.mark.parametrize("call", ["cs_cache_write", "cs_cache_read"])
def test_cache_rows_refusals(call):
    def st(**kw):
        return write_status(kw.pop("c", cache()), call=call, **kw)
    assert write_status(None, call=call) == INV
    assert st(c=cache(struct_size=8)) == INV
    assert st(c=cache(n_kv_heads=0)) == INV and st(c=cache(n_pages=0)) == INV and st(c=cache(n_pages=-1)) == INV
    assert st(c=cache(n_kv_heads=1025)) == UNS
    assert st(c=cache(head_dim=80)) == UNS and st(c=cache(page_tokens=16)) == UNS and st(c=cache(page_tokens=1 << 21)) == UNS
    assert st(c=cache(page_tokens=0)) == INV
    assert st(dtype=7) == INV and st(n=-1) == INV and st(n=1 << 31) == UNS
    assert st(n=0) == 0 and st(n=0, k=0, v=0, slots=0, pool=0) == 0
    for name in ("k", "v", "pool"):
        assert st(**{name: 0}) == INV and st(**{name: 40}) == INV
    assert st(slots=0) == INV and st(slots=12) == INV and st(err=6) == INV
    assert st(k_row=255) == INV and st(v_row=-256) == INV and st(k_row=1 << 41) == INV
    assert st(k_row=260) == UNS                                      # 520 bytes
    assert call in B.last_error()


def test_cache_query():
    with pytest.raises(B.CsError):
        B.cs_cache_query(2, 96, 32)
    assert B.lib().cs_cache_query(C.byref(cache()), None, None) == 0
    assert B.cs_cache_query(4, 128, 1 << 20, 1 << 20)[1] == 4 * (1 << 40) * 136       # past 32 bits


def batch(**kw):
    d = dict(n_seqs=2, n_queries=2, max_queries=1, table_width=3, max_keys=90, cu_queries=16, n_keys=32, page_table=64) | kw
    return B.cs_cache_batch(d.pop("struct_size", C.sizeof(B.cs_cache_batch)), **d)


def attend_status(c=None, b=None, pool=256, q=512, q_row=1024, out=1024, out_row=1024, heads=8, scale=0.1, causal=1, ws=2048, ws_bytes=1 << 40, err=None):
    return B.lib().cs_attention_cache(C.byref(c or cache()), pool, C.byref(b or batch()), q, q_row, out, out_row, heads, scale, causal, ws,
                                      ws_bytes, err, None)


def test_attention_refusals():
    L = B.lib()
    assert L.cs_attention_cache(None, 256, C.byref(batch()), 512, 1024, 1024, 1024, 8, .1, 1, 2048, 1 << 40, None, None) == INV
    assert L.cs_attention_cache(C.byref(cache()), 256, None, 512, 1024, 1024, 1024, 8, .1, 1, 2048, 1 << 40, None, None) == INV
    assert attend_status(c=cache(head_dim=256)) == UNS
    assert attend_status(b=batch(struct_size=1)) == INV
    for name in ("n_seqs", "n_queries", "max_queries", "table_width", "max_keys"):
        assert attend_status(b=batch(**{name: -1})) == INV
    assert attend_status(b=batch(max_keys=(1 << 30) + 1)) == UNS and attend_status(b=batch(n_queries=1 << 31)) == UNS
    assert attend_status(b=batch(n_queries=0)) == 0 and attend_status(b=batch(n_seqs=0)) == 0 and attend_status(b=batch(max_queries=0)) == 0
    assert attend_status(heads=7) == INV and attend_status(heads=0) == INV and attend_status(heads=2048) == UNS
    assert attend_status(causal=2) == INV
    for scale in (float("inf"), float("nan")):
        assert attend_status(scale=scale) == INV
    for name in ("pool", "q", "out"):
        assert attend_status(**{name: 0}) == INV and attend_status(**{name: 24}) == INV
    for name in ("cu_queries", "n_keys", "page_table"):
        assert attend_status(b=batch(**{name: 0})) == INV and attend_status(b=batch(**{name: 18})) == INV
    assert attend_status(q_row=1000) == INV and attend_status(out_row=1028) == UNS and attend_status(err=2) == INV
    b = batch(max_keys=5000, table_width=200)
    need = C.c_size_t()
    assert L.cs_attention_cache_query(C.byref(cache()), C.byref(b), 8, C.byref(need)) == 0 and need.value > 0
    assert attend_status(b=b, ws_bytes=need.value - 1) == WS and str(need.value) in B.last_error()
    assert attend_status(b=b, ws=0) == INV and attend_status(b=b, ws=8) == INV
    assert L.cs_attention_cache_query(C.byref(cache()), C.byref(b), 8, None) == INV
    assert L.cs_attention_cache_query(C.byref(cache()), C.byref(b), 9, C.byref(need)) == INV


def test_workspace_does_not_need_device_pointers_and_grows_with_the_keys():
    need, last = C.c_size_t(), -1
    for keys in (0, 1, 300, 4000, 100000, 1 << 30):
        b = batch(max_keys=keys, cu_queries=None, n_keys=None, page_table=None)
        assert B.lib().cs_attention_cache_query(C.byref(cache()), C.byref(b), 8, C.byref(need)) == 0
        assert need.value >= last
        last = need.value


def qk_status(q=256, k=512, qo=1024, ko=2048, row=1024, k_row=256, dtype=None, qg=64, kg=128, cs=4096, pos=16, n=3, err=None, **kw):
    d = dict(n_heads=8, n_kv_heads=2, head_dim=128, rotary_dim=128, axes=3, interleaved=0, n_positions=10, eps=1e-6) | kw
    s = d.pop("sections", (16, 24, 24))
    c = B.cs_qk_config(d.pop("struct_size", C.sizeof(B.cs_qk_config)), sections=(C.c_int32 * 3)(*s), **d)
    return B.lib().cs_qk_norm_rope(C.byref(c), q, row, k, k_row, qo, row, ko, k_row, B.CS_BF16 if dtype is None else dtype, qg, kg, cs, pos, n, err, None)


def test_qk_norm_rope_refusals():
    assert B.lib().cs_qk_norm_rope(None, *([256, 1024] * 4), B.CS_BF16, 64, 64, 64, 64, 1, None, None) == INV
    assert qk_status(struct_size=4) == INV and qk_status(dtype=3) == INV
    assert qk_status(n_heads=-1) == INV and qk_status(n_heads=0, n_kv_heads=0) == INV and qk_status(n_heads=1025) == UNS
    assert qk_status(head_dim=0) == INV and qk_status(rotary_dim=144) == INV and qk_status(head_dim=272, rotary_dim=128) == UNS
    assert qk_status(head_dim=120, rotary_dim=112, sections=(56, 0, 0)) == UNS and qk_status(rotary_dim=24, sections=(12, 0, 0)) == UNS
    assert qk_status(axes=0) == INV and qk_status(axes=4) == INV
    assert qk_status(sections=(16, 24, 23)) == INV and qk_status(sections=(-8, 36, 36)) == INV
    assert qk_status(axes=2) == INV                                   # a section of an axis that is not there
    assert qk_status(interleaved=2) == INV and qk_status(interleaved=1) == INV        # 24 of 64 pairs: more than every third
    assert qk_status(interleaved=1, axes=2, sections=(44, 20, 0)) == INV
    assert qk_status(eps=-1.0) == INV and qk_status(eps=float("nan")) == INV
    assert qk_status(n_positions=0) == INV and qk_status(n=-1) == INV and qk_status(n=1 << 31) == UNS
    assert qk_status(n=0) == 0 and qk_status(n=0, q=0, k=0, pos=0) == 0
    for name in ("q", "k", "qo", "ko", "cs"):
        assert qk_status(**{name: 0}) == INV and qk_status(**{name: 8}) == INV
    assert qk_status(pos=0) == INV and qk_status(pos=6) == INV and qk_status(err=1) == INV
    assert qk_status(qg=0) == INV and qk_status(kg=0) == INV and qk_status(qg=8) == INV
    assert qk_status(row=1020) == INV and qk_status(row=1028) == UNS and qk_status(k_row=128) == INV


def test_the_binding_refuses_what_it_cannot_describe():
    import torch
    x = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    slots = torch.zeros(4, dtype=torch.int64)
    pool = torch.zeros(2, 2 * 32 * 136, dtype=torch.uint8)
    with pytest.raises(ValueError):
        B.cs_cache_write(pool, x, x, slots, 32)                       # not on the GPU
    with pytest.raises(ValueError):
        B.cs_cache_write(pool, x, x[:, :1], slots, 32)
    with pytest.raises(ValueError):
        B.cs_cache_write(pool, x, x, slots, 64)                       # the page's size
    with pytest.raises(TypeError):
        B.cs_attention_cache(x.float(), pool, slots, slots, slots, 1, 1, 2, 32)
    with pytest.raises(ValueError):
        B.cs_qk_norm_rope(x, x[:3], torch.zeros(4, 64, 2), slots, (64,))


def test_sizes_of_a_cache_that_do_not_fit_are_refused():
    for args in (((1 << 32) + 2, 128, 32), (2, (1 << 32) + 128, 32), (2, 128, (1 << 32) + 32), (2, 128, 32, (1 << 64) + 5), (2, 128, 1 << 31)):
        with pytest.raises(ValueError, match="does not fit"):
            B.cs_cache_query(*args)
