"""What tree attention keeps of a cached key and of a projected query, and what the tests ask of it.

A rotated key is held as fp16 and the rest of it as bf8 (5 exponent and 2 fraction bits), met by the queries' leading bits (the
upper byte of an fp16 number: cut to 2 fraction bits); plain keys are met by their queries' projections as the sum of two
fp16. The usual inputs hide whether the second part is there: the roundings of weights and results are as large as what it
adds. These inputs do not: queries of elements about 200, chosen nearly orthogonal to every key, so that a logit is
the small difference of large terms, and rows that see the cache alone. A key kept as fp16 alone then puts an RMS error of
200 x 2^-11 x 0.4 = 0.04 into the logits, the weights' own rounding 2^-11 x 0.4.

Limits, of the RMS error over all rows relative to that of the first part alone. Rotated: of each term of a rest at most
1 - (1 - 2^-3) (1 - 2^-2) = 0.35 is lost (a rounding to bf8 is half a step, 2^-3; a cut to two bits loses less than 2^-2), and the
sum's RMS with it; left out the error is 1, added with the wrong sign 1.65 at least, met by another feature's query more than 1.
The limit is 0.6. Plain: two fp16 hold a projection to 2^-22 where one holds 2^-11, so what the second leaves is nothing
beside the roundings of weights and results, 2^-11 at most of each; twice these are below 0.25 of the first part's error for
these inputs (test_tree_bits.py), which is the limit."""
import math

import numpy as np
import torch

from oracle import attention as oatt

SIZE = 200.0
TOKENS = 100
ROWS = [(128, b, 64, 4) for b in (1, 2, 3, 5, 8)]
LIMIT = {True: 0.6, False: 0.25}  # rotated, plain


def bf8(x):
    return torch.as_tensor(x, dtype=torch.float32).to(torch.float8_e5m2).double().numpy()


def lead(q):
    """Queries (fp16) cut to their upper byte."""
    return (q.view(np.uint16) & np.uint16(0xFF00)).view(np.float16).astype(np.float64)


def large_queries(units, u, M, base, rng, size=SIZE):
    """M queries whose logits over the unit's keys are small differences: of elements about `size`, fp16."""
    k = units.keys(u, TOKENS, base)
    _, _, vt = np.linalg.svd(k, full_matrices=True)
    free = vt[TOKENS:]
    q = rng.standard_normal((M, 128 - TOKENS)) @ free
    q *= size / np.sqrt((q * q).mean(axis=1, keepdims=True))
    want = 1.5 * rng.standard_normal((M, TOKENS)) * math.sqrt(128)
    return (q + want @ np.linalg.pinv(k).T).astype(np.float16)


def logits(units, u, q, base, form):
    """Logits (M, TOKENS) in nats: "exact", or as kept: "first" part alone, "both", "negated" or "shuffled" (the second part met by
    another feature's query)."""
    q64 = q.astype(np.float64)
    step = float(units.delta[0][u])
    k = units.keys(u, TOKENS, base) / step
    if form == "exact":
        s = q64 @ k.T
    elif base:
        hi = k.astype(np.float16).astype(np.float64)
        rest = bf8((k - hi) * 2048) / 2048
        q8 = lead(q)
        if form == "shuffled":
            q8 = np.roll(q8, 16, axis=1)
        s = q64 @ hi.T + {"first": 0.0, "both": 1.0, "negated": -1.0, "shuffled": 1.0}[form] * (q8 @ rest.T)
    else:
        P = oatt.fp16_to_f64(units.P[0][u])
        z = oatt.dequantize(units.codes[0][u][:TOKENS], step, units.rows[u][1]) / step
        y = q64 @ P.T
        hi = y.astype(np.float16).astype(np.float64)
        lo = (y - hi).astype(np.float16).astype(np.float64)
        if form == "shuffled":
            lo = np.roll(lo, 16, axis=1)
        s = (hi + {"first": 0.0, "both": 1.0, "negated": -1.0, "shuffled": 1.0}[form] * lo) @ z.T
    return s * step / math.sqrt(128)


def attended(units, u, s):
    p = np.exp(s - s.max(axis=1, keepdims=True))
    return (p / p.sum(axis=1, keepdims=True)) @ units.values(u, TOKENS)


def other_roundings(units, u, s):
    """RMS bound of the weights' and the result's roundings to fp16, half a step each."""
    p = np.exp(s - s.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    v = units.values(u, TOKENS)
    o = p @ v
    w2 = p * p
    var = w2 @ (v * v) - 2 * o * (w2 @ v) + o * o * w2.sum(axis=1, keepdims=True)
    return 2.0 ** -11 * (math.sqrt(float(np.maximum(var, 0).mean())) + rms(o))


def rms(x):
    return float(np.sqrt((np.asarray(x) ** 2).mean()))
