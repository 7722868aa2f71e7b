"""What the calls of the verify step refuse, on the host before any launch (no GPU), and what their bindings assert."""
import ctypes

import numpy as np
import pytest

from paper_2609_24298_amd import kvc

E, U, S = kvc.KVC_EINVAL, kvc.KVC_EUNSUPPORTED, kvc.KVC_ENOSPACE
FAKE = 4096  # never dereferenced: validation fails first


class Desc:
    def __init__(self, side, n_units=2, capacity=128, r=4, b=3):
        self.keep = [np.full(n_units, r, np.int32), np.full(n_units, b, np.int32), np.arange(n_units, dtype=np.int64) * 65536,
                     np.zeros(n_units, np.int64), np.full(n_units, 0.5, np.float32)]
        p = [a.ctypes.data for a in self.keep]
        self.d = kvc.StreamDesc(n_units=n_units, d=128, capacity=capacity, side=side, r_host=p[0], b_host=p[1], code_off_host=p[2],
                                basis_off_host=p[3], delta_host=p[4], r=FAKE, b=FAKE, code_off=FAKE, basis_off=FAKE, delta=FAKE,
                                codes=FAKE, codes_bytes=1 << 40, basis=FAKE, basis_elems=1 << 20)


def tree(k=None, v=None, **kw):
    a = dict(q=FAKE, G=4, n=8, xk=FAKE, sk=1024, xv=FAKE, sv=1024, mask=FAKE, seq=FAKE, m=128, base=10000.0, out=FAKE, ws=FAKE, nb=1 << 40)
    a.update(kw)
    k, v = k or Desc(0), v or Desc(1)
    return kvc.lib().kvc_tree_attn(ctypes.byref(k.d), ctypes.byref(v.d), a["q"], a["G"], a["n"], a["xk"], a["sk"], a["xv"], a["sv"], a["mask"],
                                   a["seq"], a["m"], a["base"], a["out"], a["ws"], a["nb"], None)


@pytest.mark.parametrize("kw,code", [
    ({"G": 0}, U), ({"G": 17}, U), ({"n": 0}, U), ({"n": 65}, U), ({"m": -1}, E), ({"m": 129}, S),
    ({"base": 1.0}, E), ({"base": -5.0}, E), ({"base": float("nan")}, E), ({"base": float("inf")}, E),
    ({"q": None}, E), ({"mask": None}, E), ({"seq": None}, E), ({"out": None}, E), ({"xk": None}, E), ({"xv": None}, E), ({"ws": None}, E),
    ({"q": FAKE + 8}, E), ({"out": FAKE + 2}, E), ({"mask": FAKE + 4}, E), ({"seq": FAKE + 2}, E), ({"xk": FAKE + 8}, E),
    ({"sk": 1028}, E), ({"sk": 1016}, E), ({"sv": 8}, E), ({"ws": FAKE + 128}, E), ({"nb": 100}, S)])
def test_tree_refuses(kw, code):
    assert tree(**kw) == code
    assert kvc.lib().kvc_last_error() != b""


def test_tree_refuses_descriptors():
    assert tree(k=Desc(1)) == E and tree(v=Desc(0)) == E
    assert tree(v=Desc(1, n_units=3)) == E
    assert tree(k=Desc(0, r=5)) == U and tree(k=Desc(0, b=9)) == U
    assert tree(k=Desc(0, capacity=2 ** 31 - 1, r=128, b=8), v=Desc(1, capacity=2 ** 31 - 1)) in (U, S)
    many = [Desc(side, n_units=40, capacity=2 ** 31 - 64, r=2, b=1) for side in (0, 1)]
    assert tree(k=many[0], v=many[1], m=2 ** 31 - 64) == U  # tiles are counted in 32 bits
    one = [Desc(side, n_units=1, capacity=2 ** 31 - 1, r=2, b=1) for side in (0, 1)]
    assert tree(k=one[0], v=one[1], m=2 ** 31 - 1) == U
    assert kvc.lib().kvc_tree_attn(None, None, None, 4, 8, None, 0, None, 0, None, None, 0, 0.0, None, None, 0, None) == E


def test_tree_workspace():
    k, v, L = Desc(0, n_units=8, capacity=1 << 20), Desc(1, n_units=8, capacity=1 << 20), kvc.lib()
    need = lambda G, n, m: L.kvc_tree_attn_workspace(ctypes.byref(k.d), ctypes.byref(v.d), G, n, m)  # noqa: E731
    assert need(4, 8, 0) >= 256  # something to point at even with no cache
    assert need(4, 65, 100) == 0 and L.kvc_last_error() != b""
    for G, n, m in ((1, 1, 1), (4, 8, 1000), (16, 64, 1 << 20)):
        assert need(G, n, m) >= 8 * G * n * 528  # a chunk's partials of every row at least
    assert tree(nb=need(4, 8, 1 << 20) - 1, k=k, v=v, m=1 << 20) == S


def norm(**kw):
    a = dict(q=FAKE, sq=512, k=FAKE, sk=128, v=FAKE, sv=128, dt=kvc.F16, S=1, N=2, H=1, G=4, wq=FAKE, wk=FAKE, eps=1e-6, pos=FAKE, base=10000.0,
             qo=FAKE, ko=FAKE, kr=FAKE, vo=FAKE)
    a.update(kw)
    return kvc.lib().kvc_norm_rope(a["q"], a["sq"], a["k"], a["sk"], a["v"], a["sv"], a["dt"], a["S"], a["N"], a["H"], a["G"], a["wq"], a["wk"],
                                   a["eps"], a["pos"], a["base"], a["qo"], a["ko"], a["kr"], a["vo"], None)


@pytest.mark.parametrize("kw,code", [
    ({"dt": 3}, U), ({"dt": -1}, U), ({"S": -1}, E), ({"N": -1}, E), ({"H": 0}, E), ({"G": 0}, E), ({"H": 65536, "G": 2}, E),
    ({"eps": -1.0}, E), ({"eps": float("nan")}, E), ({"base": 0.5}, E), ({"base": float("inf")}, E), ({"pos": None}, E), ({"pos": FAKE + 2}, E),
    ({"q": None}, E), ({"qo": None}, E), ({"k": None}, E), ({"ko": None, "kr": None}, E), ({"vo": None}, E), ({"v": None}, E),
    ({"q": None, "qo": None, "k": None, "ko": None, "kr": None, "v": None, "vo": None}, E),
    ({"q": FAKE + 8}, E), ({"sq": 504}, E), ({"sk": 132}, E), ({"sk": 136, "dt": kvc.F32, "k": FAKE + 4}, E), ({"qo": FAKE + 8}, E),
    ({"wk": FAKE + 4}, E)])
def test_norm_rope_refuses(kw, code):
    assert norm(**kw) == code


def test_norm_rope_of_nothing():
    assert norm(S=0) == kvc.KVC_OK and norm(N=0) == kvc.KVC_OK


def rows(k=None, v=None, **kw):
    a = dict(xk=FAKE, sk=1024, xv=FAKE, sv=1024, m=8, rows=FAKE, t0=FAKE, n=FAKE, max_n=4)
    a.update(kw)
    k, v = k or Desc(0), v or Desc(1)
    return kvc.lib().kvc_append_rows(ctypes.byref(k.d), ctypes.byref(v.d), a["xk"], a["sk"], a["xv"], a["sv"], a["m"], a["rows"], a["t0"], a["n"],
                                     a["max_n"], None)


@pytest.mark.parametrize("kw,code", [
    ({"max_n": -1}, E), ({"m": -1}, E), ({"max_n": 129}, S), ({"m": 0}, E), ({"rows": None, "max_n": 9}, E), ({"t0": None}, E), ({"n": None}, E),
    ({"xk": None}, E), ({"xv": FAKE + 2}, E), ({"sk": 1020}, E), ({"sv": 1016}, E), ({"rows": FAKE + 2}, E), ({"t0": FAKE + 1}, E), ({"n": FAKE + 3}, E)])
def test_append_rows_refuses(kw, code):
    assert rows(**kw) == code


def test_append_rows_of_nothing_and_descriptors():
    assert rows(max_n=0) == kvc.KVC_OK
    assert rows(k=Desc(1)) == E and rows(v=Desc(0)) == E and rows(v=Desc(1, n_units=1)) == E
    assert rows(k=Desc(0, n_units=0), v=Desc(1, n_units=0)) == kvc.KVC_OK
    assert rows(k=Desc(0, n_units=65536), v=Desc(1, n_units=65536), max_n=65, m=128, sk=16384, sv=16384) == U
