"""GPU parity of kvc_append_rows: codes bit for bit those of the exact definition (the oracle's packed streams), every width
and rank, any position inside a tile, counts from none to several tiles, rows in any order; every other bit of the arena is kept."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import native as onat
from paper_2609_24298_amd import kvc

from verify_units import RANKS, Units, bits

pytestmark = pytest.mark.gpu


def expected(units, side, xb, rows, t0, n):
    """The arena after the call: the units' codes with the new tokens in place, packed by the oracle."""
    S = units.sides[side]
    arena = S.codes.cpu().numpy().copy()
    for u, w in enumerate(units.rows):
        r, b = w[2 * side], w[2 * side + 1]
        codes = units.codes[side][u].copy()
        keep = [i for i in range(int(n[u])) if 0 <= t0[u] + i < units.capacity]
        if keep:
            idx = [int(rows[u, i]) for i in keep]
            codes[[int(t0[u]) + i for i in keep]] = onat.encode_codes(units.P[side][u], units.delta[side][u], b, xb[u][idx])
        s = onat.pack(codes, r, b, side)
        arena[S.code_off_h[u]:S.code_off_h[u] + s.size] = s
    return arena


def run(units, xk, xv, rows, t0, n, given=True):
    dev = lambda a: torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32), device="cuda")  # noqa: E731
    lo = np.clip(rows, 0, xk.shape[1] - 1)
    cnt = np.clip(n, 0, rows.shape[1])
    want = [expected(units, s, bits(x), lo, t0, cnt) for s, x in ((0, xk), (1, xv))]
    kvc.kvc_append_rows(units.K, units.V, xk, xv, dev(t0), dev(n), dev(rows) if given else None)
    torch.cuda.synchronize()
    for s in (0, 1):
        got = units.sides[s].codes.cpu().numpy()
        assert np.array_equal(got, want[s]), (s, int((got != want[s]).sum()))


def tokens(U, n_rows, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(U, n_rows, 128, generator=g, device="cuda") * scale
    x[:, :, 7] *= 5
    return x.to(torch.float16)


@pytest.mark.parametrize("max_n", [1, 4, 8, 16, 17, 40, 150])
def test_every_width(max_n):
    rows = [(RANKS[i % 10], 1 + i // 8, RANKS[(3 * i + i // 10) % 10], 1 + i % 8) for i in range(64)]
    units, rng = Units(rows, 323, max_n), np.random.default_rng(max_n)
    n_rows = max_n + 3
    xk, xv = tokens(64, n_rows, 1), tokens(64, n_rows, 2)
    pick = np.stack([rng.permutation(n_rows)[:max_n] for _ in range(64)])
    n = np.array([max_n if u % 4 == 0 else int(rng.integers(0, max_n + 1)) for u in range(64)])
    t0 = np.array([int(rng.integers(0, 323 - max_n + 1)) for _ in range(64)])
    run(units, xk, xv, pick, t0, n)


@pytest.mark.parametrize("max_n", [1, 3, 8, 17, 64, 66])
@pytest.mark.parametrize("scale", [1.0, 900.0])
def test_more_units_than_the_device_has_units_of_work(max_n, scale):
    # enough units that the kernel with a wavefront per tile is chosen (up to 64 tokens) on 256 compute units, and some more
    rows = [(RANKS[i % 10], 1 + i // 8 % 8, RANKS[(3 * i + i // 10) % 10], 1 + i % 8) for i in range(259)]
    units, rng = Units(rows, 150, max_n), np.random.default_rng(max_n)
    n_rows = max_n + 2
    xk, xv = tokens(259, n_rows, 21, scale), tokens(259, n_rows, 22, scale)
    pick = np.stack([rng.integers(0, n_rows, max_n) for _ in range(259)])
    n = np.array([max_n if u % 4 == 0 else int(rng.integers(0, max_n + 1)) for u in range(259)])
    t0 = np.array([int(rng.integers(-2, 150)) for _ in range(259)])
    run(units, xk, xv, pick, t0, n)


@pytest.mark.parametrize("U,max_n", [(3, 2), (3, 20), (260, 2), (260, 20), (260, 90)])
def test_unaligned_bases(U, max_n):
    units = Units([(RANKS[i % 10], 1 + i % 8, RANKS[(i + 3) % 10], 1 + (i // 8) % 8) for i in range(U)], 120, 30, lead=5)
    rng = np.random.default_rng(30)
    xk, xv = tokens(U, max_n, 31), tokens(U, max_n, 32)
    pick = rng.integers(0, max_n, (U, max_n))
    run(units, xk, xv, pick, rng.integers(0, 120, U), rng.integers(0, max_n + 1, U))


@pytest.mark.parametrize("max_n", [5, 70])
def test_rows_repeated_and_all_of_them(max_n):
    units = Units([(84, 3, 64, 2), (128, 2, 126, 1), (18, 7, 30, 8)], 200, 5)
    xk, xv = tokens(3, max_n, 3), tokens(3, max_n, 4)
    every = np.tile(np.arange(max_n), (3, 1))
    run(units, xk, xv, every, np.array([1, 63, 100]), np.array([max_n, max_n - 1, 1]), given=False)
    units = Units([(84, 3, 64, 2), (128, 2, 126, 1), (18, 7, 30, 8)], 200, 5)
    run(units, xk, xv, every // 3, np.array([1, 63, 100]), np.array([max_n, max_n - 1, 1]))


@pytest.mark.parametrize("max_n", [6, 80])
def test_device_values_out_of_range(max_n):
    # clamped counts and row indices, positions before the stream and past the capacity left out
    lim = 2 ** 31 - 1
    units = Units([(84, 3, 64, 2)] * 7, 130, 6)
    xk, xv = tokens(7, 9, 5), tokens(7, 9, 6)
    pick = np.random.default_rng(0).integers(-4, 14, size=(7, max_n))
    pick[0, 0], pick[0, 1] = lim, -lim - 1
    run(units, xk, xv, pick, np.array([0, -3, 127, 200, -lim - 1, lim, 50]), np.array([max_n, max_n, max_n, 4, lim, lim, -lim]))


def test_strided_tokens_and_long_vectors():
    units = Units([(84, 3, 64, 2), (128, 8, 128, 8)], 130, 7)
    wide = tokens(2, 30, 8, scale=900.0)  # far past the quantizer's range, and long enough to undo the fp32 bound
    run(units, wide[:, 4:12], wide[:, 20:28], np.tile(np.arange(8)[::-1], (2, 1)), np.array([60, 3]), np.array([8, 5]))


def test_same_codes_as_encode_and_a_captured_call():
    rows = [(84, 3, 64, 2), (128, 2, 128, 2), (66, 1, 18, 4)]
    a, b = Units(rows, 300, 9), Units(rows, 300, 9)
    xk, xv = tokens(3, 40, 9), tokens(3, 40, 10)
    t0 = torch.full((3,), 77, dtype=torch.int32, device="cuda")
    n = torch.full((3,), 40, dtype=torch.int32, device="cuda")
    kvc.kvc_encode_kv(a.K, a.V, xk, xv, 77, 40)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        kvc.kvc_append_rows(b.K, b.V, xk, xv, t0, n)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(a.K.codes, b.K.codes) and torch.equal(a.V.codes, b.V.codes)
    for k in range(3):  # the replayed call reads the counts of the day
        t0.fill_(10 * k)
        n.fill_(k)
        g.replay()
        torch.cuda.synchronize()
        if k:
            kvc.kvc_encode_kv(a.K, a.V, xk, xv, 10 * k, k)
        torch.cuda.synchronize()
        assert torch.equal(a.K.codes, b.K.codes) and torch.equal(a.V.codes, b.V.codes), k
