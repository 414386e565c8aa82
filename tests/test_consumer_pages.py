"""The host's side of a layer's sequences (paper_2603_12118_amd/consumer_layer.py), with tensors on the CPU."""
import numpy as np
import pytest

from paper_2603_12118_amd.consumer_layer import PagePool


def pool(n_pages=6, sequences=2, width=4, **kw):
    return PagePool(n_pages, 32, sequences, width, "cpu", **kw)


def test_a_released_sequence_has_no_pages_anywhere():
    p = pool()
    p.reserve(0, 70)
    p.lens[0] = 70
    p.release(0)
    assert p.owned[0] == [] and p.lens[0] == 0 and sorted(p.free) == list(range(6))
    assert (p.table == -1).all()                              # (the GPU must not find another sequence's pages there)
    p.reserve(1, 90)
    assert p.table.tolist() == [[-1] * 4, p.owned[1] + [-1]]
    assert np.array_equal(p.slots(1, 31, 3), [p.owned[1][0] * 32 + 31, p.owned[1][1] * 32, p.owned[1][1] * 32 + 1])


def test_room_for_all_or_for_none():
    p = pool()
    p.reserve_all({0: 40, 1: 64})
    owned, table = [list(o) for o in p.owned], p.table.clone()
    for tokens in ({0: 96, 1: 128}, {1: 65, 0: 129}, {0: 41, 1: 129}):       # 1 + 2 of two pages left; more than four columns
        with pytest.raises(RuntimeError, match="no room"):
            p.reserve_all(tokens)
        assert p.owned == owned and len(p.free) == 2 and (p.table == table).all()
    p.reserve_all({0: 64, 1: 128})
    assert p.free == [] and p.table[1].tolist() == p.owned[1]


def test_a_limit_inside_the_last_page():
    p = pool(max_tokens=100)
    p.reserve(0, 100)
    with pytest.raises(RuntimeError, match="no room for 101 tokens"):
        p.reserve(1, 101)
    assert pool(max_tokens=1000).max_tokens == pool().max_tokens == 128
