"""Reference of the 8-bit KV cache, on the CPU: quotients and products in
numpy's fp32 (correctly rounded), attention in fp64, one (sequence, kv head) at
a time."""
from __future__ import annotations

import numpy as np
import torch

D = 128
F = np.float32
LEAST = F(2.0 ** -100)
TOP = {"e4m3": F(448.0), "int8": F(127.0)}


def e4m3(y):
    """fp32 -> the nearest E4M3 value, ties to even."""
    y = np.asarray(y, dtype=np.float64)
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
    return np.clip(np.round(y / step) * step, -448, 448)


def encode(x, fmt):
    """Block x [B][D] fp32 -> code values [B][D] (fp64), scale."""
    a = max(F(np.abs(x).max()), LEAST)
    y = x * (TOP[fmt] / a)
    assert y.dtype == F
    return (e4m3(y) if fmt == "e4m3" else np.clip(np.round(y), -127, 127).astype(np.float64)), a / TOP[fmt]


def bounds(x):
    a = max(F(np.abs(x).max()), LEAST)
    unit = F(127.0) / a
    return np.clip(np.ceil(x.max(0) * unit), -127, 127), np.clip(np.floor(x.min(0) * unit), -127, 127), a / F(127.0)


class Pair:
    """k, v: the pair's tokens [n][D] (torch, 16-bit), in order."""

    def __init__(self, k, v, fmt, block):
        self.k, self.v = k.float().numpy(), v.float().numpy()
        self.n, self.B, self.fmt = self.k.shape[0], block, fmt
        self.nb = self.n // block
        blocks = [slice(b * block, (b + 1) * block) for b in range(self.nb)]
        self.kc = [encode(self.k[s], fmt) for s in blocks]
        self.vc = [encode(self.v[s], fmt) for s in blocks]
        self.bounds = [bounds(self.k[s]) for s in blocks]

    def scores(self, q):
        """[nb] fp32: the blocks' scores for the group q [G][D] fp32."""
        out = np.full(self.nb, -np.inf, dtype=F)
        for h in range(q.shape[0]):
            a = max(F(np.abs(q[h]).max()), LEAST)
            q8 = np.round(q[h] * (F(127.0) / a)).astype(np.int64)
            for b, (hi, lo, unit) in enumerate(self.bounds):
                i = int(np.where(q8 > 0, q8 * hi.astype(np.int64), q8 * lo.astype(np.int64)).sum())
                out[b] = max(out[b], F(i) * (a / F(127.0)))
        return np.array([out[b] * self.bounds[b][2] for b in range(self.nb)], dtype=F)

    def select(self, q, num, den):
        want = min(self.nb, max(1, -(-self.nb * num // den)))
        sc = self.scores(q)
        return sorted(sorted(range(self.nb), key=lambda b: (-sc[b], b))[:want])

    def attend(self, q, scale, picked=None):
        """[G][D] fp64 over the blocks `picked` (all) and the tail; also the largest |logit|."""
        picked = range(self.nb) if picked is None else picked
        k = [self.kc[b][0] * float(self.kc[b][1]) for b in picked] + [self.k[self.nb * self.B:].astype(np.float64)]
        v = [self.vc[b][0] * float(self.vc[b][1]) for b in picked] + [self.v[self.nb * self.B:].astype(np.float64)]
        k, v = np.concatenate(k), np.concatenate(v)
        if k.shape[0] == 0:
            return np.zeros((q.shape[0], D)), 0.0
        z = q.astype(np.float64) @ k.T * scale
        p = np.exp(z - z.max(1, keepdims=True))
        return (p / p.sum(1, keepdims=True)) @ v, float(np.abs(z).max())


def bound(zmax):
    """Relative 2-norm error that an output may have.  In units of 2^-24: a
    logit of up to zmax carries the roundings of its sum, of its two scale
    factors and of its difference from the maximum, 8 with the products' sum;
    a weight the exponential's 2, its split's 4 and its scale's 2; the sums
    over tokens, by tiles and then pairwise over waves and runs, 8."""
    return 2.0 ** -24 * (16 + 8 * zmax)
