"""kvc_norm_rope where a projection holds values that are no numbers, or whose squares leave the range of fp32. Bounds as in
test_gpu_norm_rope."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_24298_amd import kvc

from test_gpu_norm_rope import D, DT, near, reference, unit_major

pytestmark = pytest.mark.gpu
S, N, KV, G = 2, 3, 2, 4


def call(x, w, eps, base, pos):
    q, k, v = x.split((KV * G * D, KV * D, KV * D), 2)
    e = lambda *s: torch.full((*s, D), 7.0, dtype=torch.float16, device="cuda")  # noqa: E731
    o = [e(S * KV, N, G), e(S * KV, N), e(S * KV, N), e(S * KV, N)]
    kvc.kvc_norm_rope(q, k, v, pos, w, w, eps, base, G, *o)
    torch.cuda.synchronize()
    return o


def inputs(dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = (torch.randn(S, N, KV * (G + 2) * D, generator=g, device="cuda", dtype=torch.float64) * scale).to(DT[dtype])
    w = 1 + 0.3 * torch.randn(D, generator=g, device="cuda")
    pos = torch.randint(0, 140000, (S, N), generator=g, device="cuda", dtype=torch.int32)
    return x, w, pos


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("base", [10000.0, 0.0])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_no_number_stays_none(dtype, base, norm, bad):
    x, w, pos = inputs(dtype, 3)
    w = w if norm else None
    clean = call(x, w, 1e-6, base, pos)
    y, hit = x.clone(), torch.zeros(S, N, KV * (G + 2), D, dtype=torch.bool, device="cuda")
    for s, n, head, i in ((0, 1, 3, 5), (1, 2, KV * G, 100), (1, 0, KV * G + KV, 64)):  # a query, a key, a value
        y[s, n, head * D + i] = bad
        hit[s, n, head, i] = True
    got = call(y, w, 1e-6, base, pos)
    if norm:  # an element reaches its whole head by the norm (values have none), and its partner by the rotation
        hit[:, :, :KV * (G + 1)] |= hit[:, :, :KV * (G + 1)].any(-1, keepdim=True)
    hq, hk, hv = (t.permute(0, 2, 1, 3).reshape(S * KV, -1, N, D).transpose(1, 2) for t in
                  (hit[:, :, :KV * G], hit[:, :, KV * G:KV * G + KV], hit[:, :, KV * G + KV:]))
    pair = lambda h: h | h.roll(64, -1) if base else h  # noqa: E731
    for t, c, h, turned in ((got[0], clean[0], pair(hq), True), (got[1], clean[1], hk[:, :, 0], False), (got[2], clean[2], pair(hk)[:, :, 0], True),
                            (got[3], clean[3], hv[:, :, 0], False)):
        assert h.any() and torch.equal(t[~h], c[~h])  # every other element as without it
        if bad != bad:
            assert t[h].isnan().all()
        elif t is got[3] or not (norm or turned):
            assert (t[h] == 65504).all()
        elif norm:  # infinity over infinity; the head's other elements become 0
            assert (t[h].isnan() | (t[h] == 0)).all() and t[h].isnan().any()
        else:
            assert (t[h].isnan() | (t[h].abs() == 65504)).all()


@pytest.mark.parametrize("dtype,scale,eps", [("fp32", 1e20, 1e-6), ("fp32", 3e37, 1e-6), ("bf16", 1e30, 1e-6), ("bf16", 1e37, 0.0), ("fp32", 1e-25, 0.0),
                                             ("fp32", 1e-37, 0.0), ("bf16", 1e-30, 1e-60), ("fp32", 1e-20, 1e-40), ("fp32", 1e-12, 0.0)])
@pytest.mark.parametrize("base", [10000.0, 0.0])
def test_squares_outside_fp32(dtype, scale, eps, base):
    x, w, pos = inputs(dtype, 4, scale)
    x[0, 0, :D] *= 1e-3  # heads of different sizes in a wavefront
    x[1, 1, D:2 * D] = 0
    x[1, 1, D] = x[0, 0, 0]  # a head of one element
    o = call(x, w, eps, base, pos)
    f = lambda a, b: x[:, :, a * D:b * D].double().cpu().numpy().reshape(S, N, b - a, D)  # noqa: E731
    wn, p, eps32 = w.double().cpu().numpy(), pos.cpu().numpy(), float(np.float32(eps))
    _, rq, mq = reference(f(0, KV * G), wn, eps32, p, base)
    pk, rk, mk = reference(f(KV * G, KV * G + KV), wn, eps32, p, base)
    near(o[0], unit_major(rq, KV), unit_major(mq, KV))
    near(o[1], unit_major(pk, KV)[:, :, 0], unit_major(mk, KV)[:, :, 0])
    near(o[2], unit_major(rk, KV)[:, :, 0], unit_major(mk, KV)[:, :, 0])


def test_small_values_beside_eps_are_as_they_were():
    # eps far above the squares: nothing to rescue, the result is x / sqrt(eps) w
    x, w, pos = inputs("fp32", 5, 1e-30)
    o = call(x, w, 1.0, 10000.0, pos)
    assert all((t == 0).all() for t in o)
