"""GPU parity of tree attention (kvc_tree_attn) where queries, keys or values are far from unit size. Bounds as in
verify_units.tree_reference."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_tree import BASE, check, draw
from tree_scales import ScaledUnits
from verify_units import half, run_tree, tree_reference

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


@pytest.mark.parametrize("N,G", TREES)
@pytest.mark.parametrize("base", [BASE, 0.0])
@pytest.mark.parametrize("e", [6, 10, 14, 20])
def test_logits_of_any_size_stay_finite(N, G, base, e):
    # queries of the longest vectors that fp16 has, keys up to 2^20: logits to 2^36. One token takes all of a row.
    units = ScaledUnits(ROWS, 300, 42, k_scale=2.0 ** e)
    q, xk, xv, words = draw(units, N, G, 42)
    q = (np.sign(q.astype(np.float32)) * 65504).astype(np.float16)
    lens = [300, 130, 64]
    got = run_tree(units, half(q), half(xk), half(xv), words, lens, 300, base).cpu().numpy().astype(np.float64)
    assert np.isfinite(got).all()
    clear = 0
    for u in range(3):
        k, v = units.keys(u, lens[u], base), units.values(u, lens[u])
        qq = q[u].astype(np.float64).reshape(N * G, 128)
        sees = np.array([[(int(words[u, n]) >> m) & 1 for m in range(N)] for n in range(N)], bool).repeat(G, axis=0)
        s = np.concatenate([qq @ k.T, np.where(sees, qq @ xk[u].astype(np.float64).T, -np.inf)], axis=1) / np.sqrt(128)
        # a logit is off by at most 2^-11 of the sum of its terms' sizes
        err = 2.0 ** -11 * (np.abs(qq) @ np.abs(k).T).max(axis=1) / np.sqrt(128)
        first = np.sort(s, axis=1)
        sure = first[:, -1] - first[:, -2] > 2 * err + 30
        want = np.concatenate([v, xv[u].astype(np.float64)])[s.argmax(axis=1)]
        e_ = np.abs(got[u].reshape(N * G, 128) - want)[sure]
        assert (e_ <= (2.0 ** -10 * np.abs(want) + 2.0 ** -18 * np.abs(want).max(axis=1, keepdims=True) + 2.0 ** -24)[sure]).all()
        clear += int(sure.sum())
    assert clear >= N * G  # a third of the rows at least


@pytest.mark.parametrize("N,G", TREES)
@pytest.mark.parametrize("base", [BASE, 0.0])
def test_results_past_fp16_become_its_largest(N, G, base):
    # values near the largest fp16 number, off by up to half a step of few bits after their reconstruction
    units = ScaledUnits(ROWS, 200, 43, v_scale=2.0 ** 17)
    q, xk, xv, words = draw(units, N, G, 43)
    xv = np.clip(xv.astype(np.float32) * 2.0 ** 15, -65504, 65504).astype(np.float16)
    words[:, -1] = 0
    lens = np.array([1, 2, 0])
    got = run_tree(units, half(q), half(xk), half(xv), words, lens, 200, base).cpu().numpy().astype(np.float64)
    past = 0
    for u in range(3):
        ref, bound = tree_reference(units, u, q[u], xk[u], xv[u], words[u], int(lens[u]), base)
        past += int((np.abs(ref) > 65504 + bound).sum())
        assert (np.abs(got[u] - np.clip(ref, -65504, 65504)) <= bound).all(), u
    assert past > 100


def test_a_row_of_no_numbers_stays_one_and_alone():
    units = ScaledUnits(ROWS, 200, 44)
    for N, G in TREES:
        for base in (BASE, 0.0):
            q, xk, xv, words = draw(units, N, G, 44)
            clean = run_tree(units, half(q), half(xk), half(xv), words, LENS, 200, base)
            q[1, N // 2, 1] = np.nan
            got = run_tree(units, half(q), half(xk), half(xv), words, LENS, 200, base)
            assert got[1, N // 2, 1].isnan().all()
            got[1, N // 2, 1] = clean[1, N // 2, 1]
            assert torch.equal(got, clean), (N, G, base)


@pytest.mark.parametrize("base", [BASE, 0.0])
@pytest.mark.parametrize("N,G", [(1, 1), (5, 4), (40, 4)])
@pytest.mark.parametrize("gap", [6.0, 12.0, 18.0])
@pytest.mark.parametrize("cached", [True, False])
def test_a_small_share_keeps_its_bits(N, G, base, gap, cached):
    # One side (cached or drafted) takes all but e^-gap of the weights and adds (next to) nothing to the result: what the other
    # gives is right to its own size. Each row sees one draft, itself; all keys of its cache are nearly alike.
    units = ScaledUnits(ROWS[:2], 130, 45, k_scale=2.0 ** -8, v_scale=2.0 ** 8 if cached else 2.0 ** -20)
    rng = np.random.default_rng(45)
    q = rng.standard_normal((2, N, G, 128)).astype(np.float16)
    q[:, :, :] = q[:, :, :1]  # a token's heads alike, so that its draft's logit is one
    q64 = q.astype(np.float64)
    lens = np.array([130, 67])
    xk = np.zeros((2, N, 128), np.float16)
    for u in range(2):
        top = (q64[u, :, 0] @ units.keys(u, lens[u], base).T).max(axis=1) + np.log(lens[u]) * np.sqrt(128)
        want = top + (gap if cached else -gap) * np.sqrt(128)
        xk[u] = (want / (q64[u, :, 0] ** 2).sum(axis=1))[:, None] * q64[u, :, 0]
    xv = np.zeros((2, N, 128), np.float16) if cached else (rng.standard_normal((2, N, 128)) * 2.0 ** 10).astype(np.float16)
    words = np.tile(np.uint64(1) << np.arange(N, dtype=np.uint64), (2, 1))
    got = run_tree(units, half(q), half(xk), half(xv), words, lens, 130, base).cpu().numpy().astype(np.float64)
    for u in range(2):
        ref, _ = tree_reference(units, u, q[u], xk[u], xv[u], words[u], int(lens[u]), base)
        size = np.abs(ref).max(axis=-1, keepdims=True)
        # weights and result to half a step of fp16 each (2^-11, of the row's largest element for sums of many, and 2^-25 where the
        # result is below 2^-14), a logit's own error by a key's rounding, 2^-12 |q * k| / sqrt(d) < 2^-12 here, and fp32's
        assert (np.abs(got[u] - ref) <= (3 * 2.0 ** -11 + 2.0 ** -12) * size + 2.0 ** -25).all(), float((np.abs(got[u] - ref) / size).max())
