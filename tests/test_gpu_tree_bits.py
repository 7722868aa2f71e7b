"""The second part of cached keys (rotated) and of projected queries (plain) reaches the logits: the RMS error of rows that only
it keeps accurate, in every form of the kernel. Inputs and limits: tree_bits."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import tree_bits as tb
from tree_scales import ScaledUnits
from verify_units import half, run_tree

pytestmark = pytest.mark.gpu


def second_parts(N, G, base, e):
    """Queries 2^-e and keys 2^e times their size."""
    U = len(tb.ROWS)
    units, rng = ScaledUnits(tb.ROWS, tb.TOKENS, 50, k_scale=2.0 ** e), np.random.default_rng(50 + N)
    q = np.stack([tb.large_queries(units, u, N * G, base, rng, tb.SIZE * 2.0 ** -e) for u in range(U)])
    none = half(np.zeros((U, N, 128), np.float16))
    got = run_tree(units, half(q.reshape(U, N, G, 128)), none, none, np.zeros((U, N), np.uint64), [tb.TOKENS] * U, tb.TOKENS, base)
    got = got.cpu().numpy().astype(np.float64).reshape(U, N * G, 128)
    for u in range(U):
        ref = tb.attended(units, u, tb.logits(units, u, q[u], base, "exact"))
        first = tb.rms(tb.attended(units, u, tb.logits(units, u, q[u], base, "first")) - ref)
        e = tb.rms(got[u] - ref) / first
        print(f"[tree bits N={N} G={G} base={base:g} b={tb.ROWS[u][1]}] {e:.3f} of the first part's error", file=sys.stderr, flush=True)
        assert e <= tb.LIMIT[bool(base)], (u, e)


@pytest.mark.parametrize("base", [500000.0, 0.0])
@pytest.mark.parametrize("N,G", [(1, 1), (5, 4), (13, 4), (25, 4), (40, 4), (64, 8)])
def test_second_parts(N, G, base):
    second_parts(N, G, base, 0)


@pytest.mark.parametrize("N,G", [(5, 4), (13, 4), (25, 4), (40, 4)])
@pytest.mark.parametrize("e", [9, 15, 18])
def test_second_parts_of_small_queries(N, G, e):
    # plain keys only: a rotated key's rest is met by what a query has of leading bits, which are fewer below 2^-14
    second_parts(N, G, 0.0, e)
