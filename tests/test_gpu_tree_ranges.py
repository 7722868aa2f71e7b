"""GPU parity of tree attention (kvc_tree_attn) where queries, keys or values are far from unit size. Bounds as in
verify_units.tree_reference."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_tree import BASE, check, draw
from tree_scales import ScaledUnits
from verify_units import half, run_tree

pytestmark = pytest.mark.gpu

ROWS = [(128, 2, 64, 2), (84, 3, 30, 4), (48, 8, 128, 1)]
TREES = [(5, 4), (13, 4), (25, 4), (40, 4)]  # rows of a wavefront and wavefronts in rows: every form of the kernel
LENS = np.array([200, 130, 64])


@pytest.mark.parametrize("N,G", TREES)
@pytest.mark.parametrize("base", [BASE, 0.0])
@pytest.mark.parametrize("e", [-8, 11, 13, 20])
def test_small_queries_and_large_keys(N, G, base, e):
    # logits as ever, of queries 2^-e and keys 2^e times their usual size
    units = ScaledUnits(ROWS, 200, 40, k_scale=2.0 ** e)
    q, xk, xv, words = draw(units, N, G, 40)
    q = (q.astype(np.float64) * 2.0 ** -e).astype(np.float16)
    xk = (xk.astype(np.float64) * 2.0 ** min(e, 13)).astype(np.float16)
    got = run_tree(units, half(q), half(xk), half(xv), words, LENS, 200, base)
    check(units, got, q, xk, xv, words, LENS, base)


@pytest.mark.parametrize("N,G", TREES)
def test_rows_of_different_sizes(N, G):
    # neighbouring rows of a wavefront differ by up to 2^10: each has a scale of its own
    units = ScaledUnits(ROWS, 200, 41, k_scale=2.0 ** 7)
    q, xk, xv, words = draw(units, N, G, 41)
    by = 2.0 ** -(4.0 + np.random.default_rng(41).integers(0, 11, (3, N, G, 1)))
    q = (q.astype(np.float64) * by).astype(np.float16)
    q[:, -1, -1] = 0
    got = run_tree(units, half(q), half(xk), half(xv), words, LENS, 200, 0.0)
    check(units, got, q, xk, xv, words, LENS, 0.0)
