"""GPU parity of tree attention (kvc_tree_attn) against fp64: every code width and rank, both forms (rotated and plain
keys), ragged lengths from none to several chunks, masks with empty rows, strides, streams and captured calls. The bound is
derived in verify_units.tree_reference."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_24298_amd import kvc

from verify_units import RANKS, Units, half, random_tree, run_tree, tree_reference

pytestmark = pytest.mark.gpu

BASE = 500000.0


def log(*a):
    print(*a, file=sys.stderr, flush=True)


def draw(units, N, G, seed, scale=2.0):
    U, rng = len(units.rows), np.random.default_rng(seed)
    norm = np.array([np.sqrt(w[0] / 128) for w in units.rows])[:, None, None]
    q = (rng.standard_normal((U, N, G, 128)) * scale / norm[..., None]).astype(np.float16)
    xk = (rng.standard_normal((U, N, 128)) * norm).astype(np.float16)
    xv = rng.standard_normal((U, N, 128)).astype(np.float16)
    words = np.stack([random_tree(rng, N, None if u % 3 else int(rng.integers(1, N + 1))) for u in range(U)])
    return q, xk, xv, words


def check(units, got, q, xk, xv, words, lens, base, which=None):
    got, worst = got.cpu().numpy().astype(np.float64), 0.0
    assert np.isfinite(got).all()
    for u in which if which is not None else range(len(units.rows)):
        ref, bound = tree_reference(units, u, q[u], xk[u], xv[u], words[u], int(lens[u]), base)
        e = np.abs(got[u] - ref) / bound
        worst = max(worst, float(e.max()))
        assert e.max() <= 1.0, (u, units.rows[u], int(lens[u]), float(e.max()))
    return worst


@pytest.fixture(scope="module")
def all_widths():
    rows = [(RANKS[i % 10], 1 + i // 8, RANKS[(3 * i + i // 10) % 10], 1 + i % 8) for i in range(64)]
    return Units(rows, 261, 3)


@pytest.mark.parametrize("N,G", [(1, 1), (5, 3), (9, 4), (5, 16), (33, 4)])
@pytest.mark.parametrize("base", [BASE, 0.0])
def test_every_width(all_widths, N, G, base):
    q, xk, xv, words = draw(all_widths, N, G, 10 * N + G)
    lens = np.array([(261, 1, 64, 65, 0, 63, 200, 128)[u % 8] for u in range(64)])
    got = run_tree(all_widths, half(q), half(xk), half(xv), words, lens, 261, base)
    worst = check(all_widths, got, q, xk, xv, words, lens, base)
    log(f"[tree widths N={N} G={G} base={base:g}] at most {worst:.2f} of the bound")


@pytest.mark.parametrize("U,N,G,T", [(1, 1, 1, 1), (3, 64, 16, 700), (2, 17, 5, 3001), (1, 64, 1, 9000), (2, 3, 2, 40000), (1, 1, 4, 130001),
                                     (40, 2, 4, 90), (3, 32, 4, 5000)])
def test_sizes(U, N, G, T):
    rows = [((128, 2, 128, 2), (84, 3, 64, 4), (64, 1, 30, 1))[u % 3] for u in range(U)]
    units = Units(rows, T, U + N)
    q, xk, xv, words = draw(units, N, G, T)
    rng = np.random.default_rng(T)
    lens = np.array([T if u == 0 else int(rng.integers(0, T + 1)) for u in range(U)])
    got = run_tree(units, half(q), half(xk), half(xv), words, lens, T, BASE)
    worst = check(units, got, q, xk, xv, words, lens, BASE, range(min(U, 3)))
    log(f"[tree U={U} N={N} G={G} T={T}] at most {worst:.2f} of the bound")


@pytest.mark.parametrize("base", [BASE, 0.0])
@pytest.mark.parametrize("N,G", [(3, 4), (13, 4), (24, 4), (40, 4)])
def test_unaligned_bases(N, G, base):
    units = Units([(84, 3, 66, 5), (128, 2, 128, 2), (18, 8, 30, 1)], 200, 15, lead=3)
    q, xk, xv, words = draw(units, N, G, 15)
    lens = np.array([200, 77, 64])
    check(units, run_tree(units, half(q), half(xk), half(xv), words, lens, 200, base), q, xk, xv, words, lens, base)


@pytest.mark.parametrize("U,N,G,T", [(3, 64, 16, 700), (2, 17, 5, 3001), (2, 3, 2, 40000), (1, 1, 4, 130001), (3, 32, 4, 5000)])
def test_sizes_of_plain_keys(U, N, G, T):
    units = Units([((128, 2, 128, 2), (84, 3, 64, 4), (64, 1, 30, 1))[u] for u in range(U)], T, U + N)
    q, xk, xv, words = draw(units, N, G, T)
    lens = np.array([T, T // 3, 64][:U])
    check(units, run_tree(units, half(q), half(xk), half(xv), words, lens, T, 0.0), q, xk, xv, words, lens, 0.0)


@pytest.fixture(scope="module")
def many_units():
    return Units([(18, 2, 14, 2)] * 2100, 200, 16)


@pytest.mark.parametrize("base", [BASE, 0.0])
@pytest.mark.parametrize("N,G", [(2, 2), (10, 4), (20, 4)])
def test_more_units_than_threads(many_units, N, G, base):
    # a thread of a block counts the tiles of several units; lengths from none to a few tiles
    units, U = many_units, 2100
    q, xk, xv, words = draw(units, N, G, 16)
    lens = np.random.default_rng(16).integers(0, 201, U)
    got = run_tree(units, half(q), half(xk), half(xv), words, lens, 200, base)
    check(units, got, q, xk, xv, words, lens, base, which=list(range(0, U, 97)) + [U - 1])


def test_sharp_and_flat_attention():
    # one key far above all others, early or late in the context, and queries near zero
    units = Units([(128, 4, 128, 4)] * 3, 2000, 8)
    q, xk, xv, words = draw(units, 6, 4, 8)
    for u, t in ((0, 3), (1, 1990)):
        k = units.keys(u, 2000, BASE)[t]
        q[u] = (k * 14 * np.sqrt(128) / (k @ k) + 0.2 * np.random.default_rng(u).standard_normal((6, 4, 128))).astype(np.float16)
    q[2] *= np.float16(1e-3)
    got = run_tree(units, half(q), half(xk), half(xv), words, [2000] * 3, 2000, BASE)
    check(units, got, q, xk, xv, words, [2000] * 3, BASE)


def test_far_logits_stay_finite():
    # logits of hundreds of nats: one token takes all of a row
    units = Units([(128, 2, 64, 2)], 500, 9)
    q, xk, xv, words = draw(units, 4, 4, 9, scale=200.0)
    got = run_tree(units, half(q), half(xk), half(xv), words, [500], 500, BASE)
    assert torch.isfinite(got).all()
    # the rounding of the keys leaves logits of this size uncertain: only finiteness is asked


@pytest.mark.parametrize("base", [BASE, 0.0])
def test_the_largest_queries_stay_finite(base):
    units = Units([(128, 2, 64, 2), (64, 8, 128, 1)], 300, 12)
    q, xk, xv, words = draw(units, 5, 4, 12)
    q = (np.sign(q.astype(np.float32)) * 65504).astype(np.float16)  # vectors of the largest norm that fp16 has
    got = run_tree(units, half(q), half(xk), half(xv), words, [300, 130], 300, base)
    assert torch.isfinite(got).all()


def test_empty_rows_and_unnamed_drafts():
    units = Units([(64, 2, 64, 2)] * 4, 100, 4)
    q, xk, xv, words = draw(units, 7, 4, 4)
    words[:] = 0
    words[1, 2] = 0b0000101   # sees drafts 0 and 2 only
    words[2, :] = [(1 << 63) | (1 << 20) | (1 << i) for i in range(7)]  # bits past the drafted tokens are ignored
    lens = np.array([0, 0, 40, 100])
    xk[0], xv[0] = np.nan, np.inf        # named by no row of their unit
    xk[1, [1, 3, 4, 5, 6]], xv[1, [1, 3, 4, 5, 6]] = np.inf, np.nan
    xk[3], xv[3] = np.nan, np.nan
    got = run_tree(units, half(q), half(xk), half(xv), words, lens, 100, BASE)
    assert (got[0] == 0).all() and (got[1, :2] == 0).all() and (got[1, 3:] == 0).all()
    check(units, got, q, np.nan_to_num(xk, posinf=0), np.nan_to_num(xv, posinf=0), words, lens, BASE)


def test_no_cache_at_all():
    units = Units([(64, 2, 64, 2)] * 2, 64, 5)
    q, xk, xv, words = draw(units, 64, 2, 5)
    got = run_tree(units, half(q), half(xk), half(xv), words, [0, 0], 0, BASE)
    check(units, got, q, xk, xv, words, [0, 0], BASE)


def test_lengths_out_of_range_are_clamped():
    units = Units([(64, 2, 64, 2)] * 3, 300, 6)
    q, xk, xv, words = draw(units, 4, 4, 6)
    args = (units, half(q), half(xk), half(xv), words)
    assert torch.equal(run_tree(*args, [-5, 100000, 250], 256, BASE), run_tree(*args, [0, 256, 250], 256, BASE))


def test_strides_ranges_and_determinism():
    units = Units([(128, 2, 64, 4), (84, 3, 126, 2), (30, 5, 18, 8), (128, 1, 128, 1)], 700, 7)
    q, xk, xv, words = draw(units, 11, 4, 7)
    wide = lambda x: half(np.concatenate([np.zeros((4, 3, 128), np.float16), x, np.full((4, 5, 128), np.nan, np.float16)], axis=1))  # noqa: E731
    lens = [700, 13, 640, 0]
    a = run_tree(units, half(q), half(xk), half(xv), words, lens, 700, BASE)
    b = run_tree(units, half(q), wide(xk)[:, 3:], wide(xv)[:, 3:], words, lens, 700, BASE)
    assert torch.equal(a, b)
    check(units, a, q, xk, xv, words, lens, BASE)
    K, V = kvc.SideRange(units.K, 1, 2), kvc.SideRange(units.V, 1, 2)
    c = run_tree(units, half(q[1:3]), half(xk[1:3]), half(xv[1:3]), words[1:3], lens[1:3], 700, BASE, K=K, V=V)
    for i in (0, 1):  # fewer units may split the context otherwise
        ref, bound = tree_reference(units, 1 + i, q[1 + i], xk[1 + i], xv[1 + i], words[1 + i], lens[1 + i], BASE)
        assert (np.abs(c[i].cpu().numpy().astype(np.float64) - ref) <= bound).all()


def test_another_stream_and_a_captured_call():
    units = Units([(128, 2, 128, 2), (64, 3, 64, 3)], 1500, 12)
    q, xk, xv, words = draw(units, 8, 4, 12)
    tq, tk, tv = half(q), half(xk), half(xv)
    lens = torch.tensor([1500, 700], dtype=torch.int32, device="cuda")
    mask = torch.as_tensor(words.view(np.int64), device="cuda")
    out = torch.empty_like(tq)
    ws = torch.empty(kvc.kvc_tree_attn_workspace(units.K, units.V, 4, 8, 1500), dtype=torch.uint8, device="cuda")
    call = lambda o, w: kvc.kvc_tree_attn(units.K, units.V, tq, 4, tk, tv, mask, lens, 1500, BASE, o, w)  # noqa: E731
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call(out, ws)
    side.synchronize()
    check(units, out, q, xk, xv, words, [1500, 700], BASE)
    g = torch.cuda.CUDAGraph()
    other, ws2 = torch.empty_like(tq), torch.empty_like(ws)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        call(other, ws2)
    for i, n in enumerate((1500, 64, 0, 999)):
        lens[0] = n
        tq.copy_(half(np.roll(q, i, axis=1)))
        other.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        call(out, ws)
        torch.cuda.synchronize()
        assert torch.equal(out, other), i
        check(units, other, np.roll(q, i, axis=1), xk, xv, words, [n, 700], BASE)
