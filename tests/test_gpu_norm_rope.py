"""GPU parity of kvc_norm_rope against fp64: types, norms, rotations, layouts by unit, absent inputs and outputs.

Bound: the rounding to fp16, half a step (2^-11 of the value, 2^-25 below 2^-14), and the fp32 work before it: the mean of squares
(a sum of 128 terms over 16 lanes, at most 12 roundings deep, halved by the root), quotient, root and two products (6 + 4 roundings
of 2^-24) and a rotation by sines and cosines within 4 2^-24 (two products, a sum: 6) of both members of a pair: 2^-19 of the
pair's magnitude covers them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_24298_amd import kvc

pytestmark = pytest.mark.gpu
D = 128
DT = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def reference(x, w, eps, pos, base):
    """x (n_seq, n_tok, heads, d) fp64 -> (normed, normed and rotated, magnitude of each value's pair)."""
    if w is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * w
    a, b = x[..., :64], x[..., 64:]
    mag = np.concatenate([np.hypot(a, b)] * 2, -1)
    if not base:
        return x, x, mag
    ang = pos[..., None, None].astype(np.float64) * base ** (-2.0 * np.arange(64) / D)
    c, s = np.cos(ang), np.sin(ang)
    return x, np.concatenate([a * c - b * s, a * s + b * c], -1), mag


def near(got, ref, mag):
    got = got.cpu().numpy().astype(np.float64)
    ref = np.clip(ref, -65504, 65504)
    assert got.shape == ref.shape
    e = np.abs(got - ref)
    lim = 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 + 2.0 ** -19 * mag
    assert np.isfinite(got).all() and (e <= lim).all(), float((e / lim).max())


def unit_major(y, kv):
    """(n_seq, n_tok, kv * g, d) -> (n_seq * kv, n_tok, g, d)"""
    S, N, H, _ = y.shape
    return y.reshape(S, N, kv, H // kv, D).transpose(0, 2, 1, 3, 4).reshape(S * kv, N, H // kv, D)


def run(S, N, kv, G, dtype, norm, base, seed=0, scale=1.0, pos=None, stream=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    H = kv * G
    x = (torch.randn(S, N, (H + 2 * kv) * D, generator=g, device="cuda") * scale).to(DT[dtype])
    q, k, v = x.split((H * D, kv * D, kv * D), 2)
    w = [(1 + 0.3 * torch.randn(D, generator=g, device="cuda")) if norm else None for _ in range(2)]
    if pos is None:
        pos = torch.randint(0, 140000, (S, N), generator=g, device="cuda", dtype=torch.int32)
    e = lambda *s: torch.full((*s, D), float("nan"), dtype=torch.float16, device="cuda")  # noqa: E731
    o = [e(S * kv, N, G), e(S * kv, N), e(S * kv, N), e(S * kv, N)]
    kvc.kvc_norm_rope(q, k, v, pos, w[0], w[1], 1e-6, base, G, *o, stream=stream)
    torch.cuda.synchronize()
    f = lambda t, h: t.double().cpu().numpy().reshape(S, N, h, D)  # noqa: E731
    wn = [None if t is None else t.double().cpu().numpy() for t in w]
    p = pos.cpu().numpy()
    _, rq, mq = reference(f(q, H), wn[0], 1e-6, p, base)
    pk, rk, mk = reference(f(k, kv), wn[1], 1e-6, p, base)
    near(o[0], unit_major(rq, kv), unit_major(mq, kv))
    one = lambda y: unit_major(y, kv)[:, :, 0]  # noqa: E731
    near(o[1], one(pk), one(mk))
    near(o[2], one(rk), one(mk))
    near(o[3], one(f(v, kv)), np.zeros(()))
    return (q, k, v, pos, w), o


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 0.0])
def test_types_norms_and_bases(dtype, norm, base):
    run(3, 7, 4, 4, dtype, norm, base)


@pytest.mark.parametrize("S,N,kv,G", [(1, 1, 1, 1), (1, 1, 8, 4), (2, 61, 8, 8), (1, 3, 5, 3), (5, 1, 2, 16), (2, 257, 3, 1), (1, 1500, 8, 4)])
def test_sizes(S, N, kv, G):
    run(S, N, kv, G, "bf16", True, 500000.0, seed=N)


def test_positions_far_and_negative():
    pos = torch.tensor([[0, 1, 2 ** 31 - 1, -2 ** 31, -1, 10 ** 9]], dtype=torch.int32, device="cuda")
    run(1, 6, 2, 2, "fp32", True, 10000.0, pos=pos)


def test_small_and_large_values():
    run(2, 5, 2, 4, "fp32", True, 10000.0, scale=1e-4)
    run(2, 5, 2, 4, "fp32", True, 10000.0, scale=1e15)
    run(2, 5, 2, 4, "fp32", False, 10000.0, scale=4e4)  # saturates
    run(2, 5, 2, 4, "bf16", False, 0.0, scale=1e6)


def test_zero_rows_and_no_tokens():
    z = torch.zeros(1, 2, 2 * D, dtype=torch.float16, device="cuda")
    w = torch.ones(D, device="cuda")
    o = torch.full((1, 2, 2, D), float("nan"), dtype=torch.float16, device="cuda")
    pos = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    kvc.kvc_norm_rope(z, None, None, pos, w, None, 1e-6, 10000.0, 2, o, None, None, None)
    assert (o == 0).all()
    kvc.kvc_norm_rope(z[:, :0], None, None, pos[:, :0], w, None, 1e-6, 10000.0, 2, o[:, :0], None, None, None)


def test_parts_alone_equal_the_whole():
    (q, k, v, pos, w), o = run(2, 9, 4, 2, "bf16", True, 500000.0, seed=3)
    for i in range(4):
        part = [torch.full_like(t, float("nan")) if j == i else None for j, t in enumerate(o)]
        kvc.kvc_norm_rope(q if i == 0 else None, k if i in (1, 2) else None, v if i == 3 else None, pos, *w, 1e-6, 500000.0, 2, *part)
        torch.cuda.synchronize()
        assert torch.equal(part[i], o[i]), i


def test_another_stream_and_a_captured_call():
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        (q, k, v, pos, w), o = run(2, 9, 4, 2, "bf16", True, 500000.0, seed=4)
    mine = [torch.empty_like(t) for t in o]
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        kvc.kvc_norm_rope(q, k, v, pos, *w, 1e-6, 500000.0, 2, *mine)
    for i in range(3):
        pos.add_(i)
        kvc.kvc_norm_rope(q, k, v, pos, *w, 1e-6, 500000.0, 2, *o)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(mine, o)), i
