"""The workspace of tree attention as a server keeps it (host only): a size taken for the largest call serves every smaller one."""
import ctypes

import pytest

from paper_2609_24298_amd import kvc

from test_verify_refusals import FAKE, S, Desc, tree


def need(k, v, G, n, m):
    return kvc.lib().kvc_tree_attn_workspace(ctypes.byref(k.d), ctypes.byref(v.d), G, n, m)


@pytest.mark.parametrize("units,capacity", [(1, 64), (1, 1 << 20), (3, 4096), (8, 1 << 20), (64, 300), (700, 32768)])
def test_never_falls_with_tokens_heads_or_length(units, capacity):
    k, v = Desc(0, n_units=units, capacity=capacity), Desc(1, n_units=units, capacity=capacity)
    lengths = sorted({0, 1, 63, 64, 65, 128, 129, capacity // 7, capacity // 2, capacity - 1, capacity} & set(range(capacity + 1)))
    for m in lengths:
        table = [[need(k, v, G, n, m) for n in range(1, 65)] for G in range(1, 17)]
        for row in table:
            assert all(0 < a <= b for a, b in zip(row, row[1:])), m
        for row, more in zip(table, table[1:]):
            assert all(a <= b for a, b in zip(row, more)), m
    for G, n in ((1, 1), (4, 16), (4, 17), (5, 13), (8, 33), (16, 64)):
        sizes = [need(k, v, G, n, m) for m in lengths]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), (G, n)
    # the call asks for what the query says
    assert tree(k=k, v=v, G=4, n=16, m=capacity, sk=2048, sv=2048, nb=need(k, v, 4, 16, capacity) - 1) == S


def test_never_falls_with_units():
    sides = [(Desc(0, n_units=n, capacity=4096), Desc(1, n_units=n, capacity=4096)) for n in (1, 2, 3, 8, 50, 51, 64, 200, 1000)]
    for G, n, m in ((1, 1, 1), (4, 16, 4096), (4, 17, 4096), (16, 64, 300), (5, 13, 0)):
        sizes = [need(k, v, G, n, m) for k, v in sides]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), (G, n, m)
