"""Batches whose launches would be larger than a grid may be (2^32 - 1 threads, workgroups of 256) are refused before anything is enqueued,
without a GPU: pointers here are plain numbers."""
import ctypes as C

import pytest

from paper_2603_12118_amd import binding as B

MOST = (2 ** 32 - 1) // 256


def status(n_seqs, n_queries, max_queries, max_keys, heads=8, kv_heads=8):
    """(of the query, of the call)"""
    c = B.cs_cache_config(C.sizeof(B.cs_cache_config), kv_heads, 64, 32, 4)
    b = B.cs_cache_batch(C.sizeof(B.cs_cache_batch), n_seqs=n_seqs, n_queries=n_queries, max_queries=max_queries, table_width=100, max_keys=max_keys,
                         cu_queries=16, n_keys=32, page_table=64)
    need = C.c_size_t()
    return (B.lib().cs_attention_cache_query(C.byref(c), C.byref(b), heads, C.byref(need)),
            B.lib().cs_attention_cache(C.byref(c), 256, C.byref(b), 512, heads * 64, 1024, heads * 64, heads, .1, 1, 2048, 1 << 62, None, None))


@pytest.mark.parametrize("args", [
    (MOST // 8 + 1, MOST // 8 + 1, 1, 500),                       # one workgroup a sequence and head
    (MOST // 8 + 1, MOST // 8 + 1, 1, 5000),                      # ... with keys that are shared out
    (131072, 131072 * 600, 1024, 500),                            # 32 blocks of rows a sequence may have
    (1 << 22, (1 << 22) + 4096, 4096, 5000),                      # prompts and tokens: the launch of the tokens, the second one
    (1 << 22, (1 << 22) + 4096, 4096, 500),
    (0x7fffffff, 0x7fffffff, 0x7fffffff, 1 << 30),
    (0x7fffffff, 0x7fffffff, 1, 500),
])
def test_refused(args):
    st = status(*args)
    assert st == (B.CS_ERR_UNSUPPORTED, B.CS_ERR_UNSUPPORTED), st
    assert "cs_attention_cache" in B.last_error()
