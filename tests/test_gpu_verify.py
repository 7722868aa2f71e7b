"""GPU parity of the verify step as a model runs it: per layer, the projections of a tree of drafted tokens are normalised,
rotated and laid out (kvc_norm_rope), attended over the cache and themselves (kvc_tree_attn), and after the last layer every
layer's accepted path is appended (kvc_append_rows), each sequence with a length of its own. Every step's outputs are held
against fp64 over the exactly defined codes (bounds of verify_units and of the norm's tests), the code streams bit for bit
against the oracle's, and a captured step, replayed, against the eager one bit for bit."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention as oatt
from oracle import native as onat
from paper_2609_24298_amd import kvc, pipeline, synth

from oracle_stats import oracle_stats
from test_gpu_norm_rope import near, reference, unit_major
from verify_units import bits, random_tree, tree_reference

pytestmark = pytest.mark.gpu
D, BASE, EPS = 128, 500000.0, 1e-6


class Codes:
    """The cache's codes by the oracle, in the form tree_reference reads them."""

    def __init__(self, cache):
        self.c, n = cache, cache.w.n_units
        self.codes = [[np.zeros((0, int(s.r_h[u])), np.uint8) for u in range(n)] for s in (cache.K, cache.V)]
        basis = [bits(s.basis) for s in (cache.K, cache.V)]
        self.P = [[basis[i][int(s.basis_off_h[u]):][:int(s.r_h[u]) * D].reshape(-1, D) for u in range(n)]
                  for i, s in enumerate((cache.K, cache.V))]

    def append(self, side, u, x):
        s = (self.c.K, self.c.V)[side]
        if len(x):
            new = onat.encode_codes(self.P[side][u], np.float32(s.delta_h[u]), int(s.b_h[u]), np.ascontiguousarray(x))
            self.codes[side][u] = np.concatenate([self.codes[side][u], new])

    def arena_equal(self, side):
        s = (self.c.K, self.c.V)[side]
        got = s.codes.cpu().numpy()
        for u, c in enumerate(self.codes[side]):
            full = np.zeros((s.capacity, c.shape[1]), np.uint8)
            full[:len(c)] = c
            want = onat.pack(full, int(s.r_h[u]), int(s.b_h[u]), side)
            off = int(s.code_off_h[u])
            assert np.array_equal(got[off:off + want.size], want), (side, u)

    def at(self, side, u, n):
        s = (self.c.K, self.c.V)[side]
        return oatt.reconstruct(self.codes[side][u][:n], self.P[side][u], float(s.delta_h[u]), int(s.b_h[u]))

    def keys(self, u, n, base):
        k = self.at(0, u, n)
        return oatt.rope_rotate(k, np.arange(n), base) if base else k

    def values(self, u, n):
        return self.at(1, u, n)


class Step:
    """A model's state between its layers: buffers of a verify step of N tokens."""

    def __init__(self, cache, N, base, max_len):
        w = cache.w
        self.c, self.N, self.base, self.max_len = cache, N, base, max_len
        self.upl = w.batch * w.kv_heads
        self.sides = [cache.layer_sides(layer) for layer in range(w.layers)]
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
        f16 = lambda *s: torch.full((*s, D), float("nan"), dtype=torch.float16, device="cuda")  # noqa: E731
        self.x = torch.zeros(w.layers, w.batch, N, (w.kv_heads * (w.group + 2)) * D, dtype=torch.bfloat16, device="cuda")
        self.wq, self.wk = torch.ones(D, device="cuda"), torch.ones(D, device="cuda")
        self.pos, self.mask = i32(w.batch, N), torch.zeros(w.n_units, N, dtype=torch.int64, device="cuda")
        self.lens, self.n, self.rows = i32(w.n_units), i32(w.n_units), i32(w.n_units, N)
        self.q, self.out = f16(w.n_units, N, w.group), f16(w.n_units, N, w.group)
        self.k, self.kr, self.v = f16(w.n_units, N), f16(w.n_units, N), f16(w.n_units, N)
        self.ws, _ = cache.verify_buffers(N, max_len, self.sides[0])

    def run(self):
        w, upl = self.c.w, self.upl
        for layer in range(w.layers):
            u = slice(layer * upl, (layer + 1) * upl)
            q, k, v = self.x[layer].split((w.kv_heads * w.group * D, w.kv_heads * D, w.kv_heads * D), 2)
            kvc.kvc_norm_rope(q, k, v, self.pos, self.wq, self.wk, EPS, self.base, w.group, self.q[u], self.k[u], self.kr[u], self.v[u])
            self.c.verify(self.q[u], self.kr[u], self.v[u], self.mask[u], self.lens[u], self.max_len, self.out[u], self.ws,
                          self.base, self.sides[layer])
        # which tokens are accepted is known after the last layer
        self.c.accept(self.k, self.v, self.lens, self.n, self.rows)
        self.lens += self.n


def draw(step, rng, g):
    """Another step's inputs: a tree per sequence, its tokens at their depths' positions, a path from a root accepted."""
    w, N = step.c.w, step.N
    step.x.copy_(torch.randn(step.x.shape, generator=g, device="cuda"))
    lens = step.lens.view(w.layers, w.batch, w.kv_heads)[0, :, 0].cpu().numpy()
    pos, mask, rows, n = [], [], [], []
    for b in range(w.batch):
        words = random_tree(rng, N, None if b % 2 == 0 else max(1, N - 2))
        depth = np.array([max(bin(int(x)).count("1") - 1, 0) for x in words])
        leaf = int(rng.integers(0, N))
        path = [m for m in range(N) if int(words[leaf]) >> m & 1]  # a leaf of a padding row accepts nothing
        pos.append(lens[b] + depth)
        mask.append(words.view(np.int64))
        n.append(len(path))
        rows.append(path + [0] * (N - len(path)))
    up = lambda a: np.broadcast_to(np.asarray(a)[None, :, None], (w.layers, w.batch, w.kv_heads) + np.shape(a)[1:])  # noqa: E731
    step.pos.copy_(torch.as_tensor(np.asarray(pos, np.int32)))
    for t, a in ((step.mask, mask), (step.rows, rows), (step.n, n)):
        t.copy_(torch.as_tensor(np.ascontiguousarray(up(a))).reshape(t.shape).to(t.dtype))
    return np.asarray(mask).view(np.uint64)


@pytest.fixture(scope="module")
def world():
    w = synth.Workload("verify_l2_h2_g4", 2, 2, 4, 3, 400, 2.0)
    return w, oracle_stats(w, 5)


def prefill(cache, w, lens):
    """Every sequence its own length: a call of chosen rows may be as long as the cache."""
    xk = pipeline.draw_unit_tokens(w, cache.stats, kvc.SIDE_K, int(lens.max()), 6, "cuda")
    xv = pipeline.draw_unit_tokens(w, cache.stats, kvc.SIDE_V, int(lens.max()), 6, "cuda")
    per = torch.as_tensor(np.tile(np.repeat(lens, w.kv_heads), w.layers).astype(np.int32), device="cuda")
    cache.accept(xk, xv, torch.zeros_like(per), per)
    return bits(xk), bits(xv), per


@pytest.mark.parametrize("N", [1, 6, 19])
@pytest.mark.parametrize("base", [BASE, 0.0])
def test_a_run_of_steps(world, N, base):
    w, st = world
    cache = pipeline.Cache(w, seed=5, stats=st, capacity=w.tokens)
    lens = np.array([0, 61, 330])
    bk, bv, per = prefill(cache, w, lens)
    codes, step = Codes(cache), Step(cache, N, base, w.tokens)
    step.lens.copy_(per)
    for u in range(w.n_units):
        codes.append(0, u, bk[u, :int(per[u])])
        codes.append(1, u, bv[u, :int(per[u])])
    rng, g = np.random.default_rng(N), torch.Generator(device="cuda")
    g.manual_seed(N)
    step.wq.copy_(1 + 0.2 * torch.randn(D, generator=g, device="cuda"))
    step.wk.copy_(1 + 0.2 * torch.randn(D, generator=g, device="cuda"))
    H = w.kv_heads
    for _ in range(3):
        words = draw(step, rng, g)
        before = step.lens.cpu().numpy().copy()
        step.run()
        torch.cuda.synchronize()
        pos, wq, wk = step.pos.cpu().numpy(), step.wq.double().cpu().numpy(), step.wk.double().cpu().numpy()
        for layer in range(w.layers):
            us = slice(layer * step.upl, (layer + 1) * step.upl)
            x = step.x[layer].double().cpu().numpy().reshape(w.batch, N, -1, D)
            _, rq, mq = reference(x[:, :, :H * w.group], wq, EPS, pos, base)
            pk, rk, mk = reference(x[:, :, H * w.group:H * (w.group + 1)], wk, EPS, pos, base)
            near(step.q[us], unit_major(rq, H), unit_major(mq, H))
            near(step.k[us], unit_major(pk, H)[:, :, 0], unit_major(mk, H)[:, :, 0])
            near(step.kr[us], unit_major(rk, H)[:, :, 0], unit_major(mk, H)[:, :, 0])
            near(step.v[us], unit_major(x[:, :, H * (w.group + 1):], H)[:, :, 0], np.zeros(()))
        q, kr, v = (t.cpu().numpy() for t in (step.q, step.kr, step.v))
        out = step.out.cpu().numpy().astype(np.float64)
        for u in range(w.n_units):
            ref, bound = tree_reference(codes, u, q[u], kr[u], v[u], words[u // H % w.batch], int(before[u]), base)
            e = np.abs(out[u] - ref)
            assert np.isfinite(out[u]).all() and (e <= bound).all(), (u, float((e / bound).max()))
        kb, vb, rows, n = bits(step.k), bits(step.v), step.rows.cpu().numpy(), step.n.cpu().numpy()
        for u in range(w.n_units):
            codes.append(0, u, kb[u, rows[u, :n[u]]])
            codes.append(1, u, vb[u, rows[u, :n[u]]])
        assert np.array_equal(step.lens.cpu().numpy(), before + n)
        codes.arena_equal(0)
        codes.arena_equal(1)


def test_a_captured_step_replayed(world):
    w, st = world
    A = pipeline.Cache(w, seed=5, stats=st, capacity=w.tokens)
    B = pipeline.Cache(w, seed=5, stats=st, capacity=w.tokens)
    lens = np.array([5, 0, 200])
    a, b = Step(A, 7, BASE, w.tokens), Step(B, 7, BASE, w.tokens)
    for c, s in ((A, a), (B, b)):
        s.lens.copy_(prefill(c, w, lens)[2])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b.run()
    torch.cuda.synchronize()
    for i in range(4):
        for s in (a, b):
            g = torch.Generator(device="cuda")
            g.manual_seed(50 + i)
            draw(s, np.random.default_rng(70 + i), g)
        a.run()
        graph.replay()
        torch.cuda.synchronize()
        for f in ("q", "k", "kr", "v", "out", "lens"):
            assert torch.equal(getattr(a, f), getattr(b, f)), (i, f)
        assert torch.equal(A.K.codes, B.K.codes) and torch.equal(A.V.codes, B.V.codes), i
    assert math.isfinite(float(a.out.float().abs().max()))
