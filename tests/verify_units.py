"""Small caches and fp64 references for the tests of the verify step (norm and rotation, tree attention, appending)."""
import math

import numpy as np
import torch

from oracle import attention as oatt
from oracle import native as onat
from paper_2609_24298_amd import kvc

RANKS = (2, 6, 14, 18, 48, 64, 66, 84, 126, 128)


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def half(a):
    return torch.as_tensor(np.asarray(a, dtype=np.float16).view(np.int16), device="cuda").view(torch.float16)


class Units:
    """Units of both sides with given (r_K, b_K, r_V, b_V), random bases, and codes of coordinates of about unit variance."""

    def __init__(self, rows, capacity, seed, device="cuda", lead=0):
        self.rows, self.capacity = rows, capacity
        rng = np.random.default_rng(seed)
        self.P, self.delta, self.codes, self.sides = ([], []), ([], []), ([], []), []
        for side in (kvc.SIDE_K, kvc.SIDE_V):
            rs, bs = [w[2 * side] for w in rows], [w[2 * side + 1] for w in rows]
            for r, b in zip(rs, bs):
                q, _ = np.linalg.qr(rng.standard_normal((128, 128)))
                self.P[side].append(q[:r].astype(np.float16).view(np.uint16))
                self.delta[side].append(np.float32(rng.uniform(0.7, 1.3) * 2.2 / 2 ** (b - 1)))
                y = rng.standard_normal((capacity, r)) * 2 ** (b - 1) / 2.2
                self.codes[side].append(np.clip(np.floor(y) + 2 ** (b - 1), 0, 2 ** b - 1).astype(np.uint8))
            gap = np.full(lead, 0x7E00, np.uint16)  # elements before each basis (NaN), so that none need be aligned
            flat = np.concatenate([x for p in self.P[side] for x in (gap, p.reshape(-1))])
            offs = np.concatenate([[0], np.cumsum([p.size + lead for p in self.P[side]])[:-1]]).astype(np.int64) + lead
            S = kvc.Side(side, rs, bs, np.array(self.delta[side], np.float32), flat, offs, capacity, device)
            arena = np.zeros(S.codes.numel(), np.uint8)
            for u, (r, b) in enumerate(zip(rs, bs)):
                s = onat.pack(self.codes[side][u], r, b, side)
                arena[S.code_off_h[u]:S.code_off_h[u] + s.size] = s
            S.codes.copy_(torch.as_tensor(arena))
            self.sides.append(S)

    @property
    def K(self):
        return self.sides[0]

    @property
    def V(self):
        return self.sides[1]

    def keys(self, u, n, base):
        k = oatt.reconstruct(self.codes[0][u][:n], self.P[0][u], float(self.delta[0][u]), self.rows[u][1])
        return oatt.rope_rotate(k, np.arange(n), base) if base else k

    def values(self, u, n):
        return oatt.reconstruct(self.codes[1][u][:n], self.P[1][u], float(self.delta[1][u]), self.rows[u][3])


def tree_reference(units, u, q, xk, xv, words, n, base):
    """fp64 rows of unit u and the bound on what the kernel's rows may differ by. q (N, G, d), xk and xv (N, d) fp16 arrays.

    Roundings, each at most half a step: of every weight to fp16, 2^-11 of it, and below 2^-14 of the largest 2^-25 of that; of
    every coordinate of a rotated cached key, whose rest after fp16 (2^-11 of it) is taken from its bf8 part (2^-3 off) times the
    query cut to two fraction bits (2^-2 off), so that less than half of it is lost: a logit moves by 2^-12 |q * k_t| / sqrt(d)
    (2-norm of the elementwise product: the signs do not line up). These move the output by the root of the sum of squares of
    w_t (v_t - o), of which eight are allowed, since half a step is the most that a rounding moves; the result's own rounding is
    added, 2^-11 of it and 2^-25 below 2^-14. fp32 sums, angles (fp64, and rotations of at most 32 steps of 2^-23 in between) and
    the two-part projection are below 2^-18 of the same terms."""
    N, G, d = q.shape
    q = q.astype(np.float64).reshape(N * G, d)
    k, v = units.keys(u, n, base), units.values(u, n)
    sees = np.array([[(int(words[i]) >> m) & 1 for m in range(N)] for i in range(N)], bool).repeat(G, axis=0)
    named = sees.any(axis=0)
    xk = np.where(named[:, None], xk.astype(np.float64), 0.0)
    xv = np.where(named[:, None], xv.astype(np.float64), 0.0)
    s = np.concatenate([q @ k.T, np.where(sees, q @ xk.T, -np.inf)], axis=1) / math.sqrt(d)
    top = s.max(axis=1, keepdims=True)
    top[np.isinf(top)] = 0.0
    p = np.exp(s - top)
    p /= np.maximum(p.sum(axis=1, keepdims=True), 1e-300)
    vals = np.concatenate([v, xv])
    o = p @ vals
    ds = np.concatenate([2.0 ** -12 * np.sqrt((q * q) @ (k * k).T) / math.sqrt(d), np.zeros((N * G, N))], axis=1)
    w2 = (p * ds) ** 2 + (2.0 ** -11 * p) ** 2 + np.where(p > 0, (2.0 ** -25 * p.max(axis=1, keepdims=True)) ** 2, 0.0)
    var = w2 @ (vals * vals) - 2 * o * (w2 @ vals) + o * o * w2.sum(axis=1, keepdims=True)
    bound = 8 * np.sqrt(np.maximum(var, 0.0)) + 2.0 ** -11 * np.abs(o) + 2.0 ** -25 + 2.0 ** -18 * np.abs(vals).max(initial=0.0)
    return o.reshape(N, G, d), bound.reshape(N, G, d)


def random_tree(rng, n, size=None):
    """Ancestor words of a random tree; rows from `size` on are empty."""
    words = np.zeros(n, np.uint64)
    for i in range(n if size is None else size):
        parent = int(rng.integers(max(-1, i - 5), i)) if i else -1
        words[i] = np.uint64(1 << i) | (words[parent] if parent >= 0 else np.uint64(0))
    return words


def run_tree(units, q, xk, xv, words, lens, max_len, base, stream=None, K=None, V=None):
    K, V = K or units.K, V or units.V
    U, N, G, _ = q.shape
    out = torch.full((U, N, G, 128), float("nan"), dtype=torch.float16, device="cuda")
    ws = torch.empty(kvc.kvc_tree_attn_workspace(K, V, G, N, max_len), dtype=torch.uint8, device="cuda")
    ws.random_(0, 256)
    kvc.kvc_tree_attn(K, V, q, G, xk, xv, torch.as_tensor(words.view(np.int64), device="cuda"),
                      torch.as_tensor(np.asarray(lens, np.int32), device="cuda"), max_len, base, out, ws, stream)
    return out
