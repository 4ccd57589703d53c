"""Reference of the 4-bit KV cache, on the CPU: grids and codes in numpy's fp32
(correctly rounded), attention in fp64, one (sequence, kv head) at a time."""
from __future__ import annotations

import numpy as np
import torch

D = 128
F = np.float32
LEAST = {torch.float16: F(2.0 ** -19), torch.bfloat16: F(2.0 ** -100)}


def round_down(y, dt):
    """The largest value of the type that is not above y >= 0 (fp32)."""
    t = torch.from_numpy(np.ascontiguousarray(y)).to(dt)
    up = t.float().numpy() > y
    return torch.where(torch.from_numpy(up), (t.view(torch.int16) - 1).view(dt), t).float().numpy()


def encode(x, dt):
    """Rows x [rows][n] fp32 (16-bit values) -> codes, scales, zeros; all fp32."""
    lo, hi = x.min(1), x.max(1)
    scale = np.maximum(round_down((hi * F(0.5) - lo * F(0.5)) / F(7.5), dt), LEAST[dt])
    code = np.rint((x * F(0.5) - (lo * F(0.5))[:, None]) * (F(2.0) / scale)[:, None])
    assert code.dtype == F and scale.dtype == F and code.min() >= 0 and code.max() <= 15
    return code, scale, lo


def values(code, scale, zero):
    """What codes stand for, in fp32 (one rounding: the product is exact)."""
    return (zero.astype(np.float64) + scale.astype(np.float64) * code.astype(np.float64)).astype(F)


class Pair:
    """k, v: the pair's tokens [n][D] (torch, 16-bit), in order."""

    def __init__(self, k, v, block):
        self.dt, self.B = k.dtype, block
        self.k, self.v = k.float().numpy(), v.float().numpy()
        self.n, self.nb = k.shape[0], k.shape[0] // block
        blocks = [slice(b * block, (b + 1) * block) for b in range(self.nb)]
        self.kc = [encode(self.k[s].T.copy(), self.dt) for s in blocks]    # codes [D][B]
        self.vc = [encode(self.v[s], self.dt) for s in blocks]             # codes [B][D]

    def held(self):
        """The tokens as the codes stand for them, in fp64 without a rounding."""
        def one(parts, raw, turn):
            whole = [z[:, None].astype(np.float64) + s[:, None].astype(np.float64) * c for c, s, z in parts]
            whole = [w.T if turn else w for w in whole]
            return np.concatenate(whole + [raw[self.nb * self.B:].astype(np.float64)])
        return one(self.kc, self.k, True), one(self.vc, self.v, False)

    def read(self):
        """The tokens as they are read back (torch, 16-bit)."""
        def one(parts, raw, turn):
            whole = [values(c, s[:, None], z[:, None]) for c, s, z in parts]
            whole = [w.T if turn else w for w in whole]
            return torch.from_numpy(np.concatenate(whole + [raw[self.nb * self.B:]])).to(self.dt)
        return one(self.kc, self.k, True), one(self.vc, self.v, False)

    def spread(self):
        """[n][D]: how large the terms of a key's and a value's products are."""
        def one(parts, raw, turn):
            whole = [np.abs(z.astype(np.float64))[:, None] + 31.0 * s.astype(np.float64)[:, None] + 0 * c for c, s, z in parts]
            whole = [w.T if turn else w for w in whole]
            return np.concatenate(whole + [np.abs(raw[self.nb * self.B:])]).astype(np.float64)
        return one(self.kc, self.k, True), one(self.vc, self.v, False)

    def decode(self, q, scale):
        """[G][D] fp64, and how far an output may be from it.  In units of 2^-24 a
        logit carries the roundings of its sum, whose terms have the root sum
        square a, and the weights' and sums' own; terms of the outputs' sums are
        up to |zero| + 31 scales."""
        q = q.astype(np.float64)
        if self.n == 0:
            return np.zeros((q.shape[0], D)), 0.0
        k, v = self.held()
        ka, va = self.spread()
        z = q @ k.T * scale
        p = np.exp(z - z.max(1, keepdims=True))
        a = abs(scale) * np.sqrt((q * q) @ (ka * ka).T).max()
        return (p / p.sum(1, keepdims=True)) @ v, 2.0 ** -24 * (16 + 16 * a) * va.max()

    def attend(self, q, scale, last):
        """Rows q [rows][D], each up to token `last` [rows] of those read back:
        [rows][D] fp64, and how far each output may be from it: a rounding of it,
        one of each weight, and the fp32 sums'."""
        q = q.astype(np.float64)
        half = torch.finfo(self.dt).eps / 2
        if self.n == 0:
            return np.zeros(q.shape), np.zeros(q.shape)
        k, v = (t.double().numpy() for t in self.read())
        z = q @ k.T * scale
        z[np.arange(self.n)[None] > np.asarray(last)[:, None]] = -np.inf
        top = z.max(1, keepdims=True)
        p = np.exp(z - np.where(np.isfinite(top), top, 0.0))
        total = p.sum(1, keepdims=True)
        p = np.divide(p, total, out=np.zeros_like(p), where=total > 0)
        a = abs(scale) * np.sqrt((q * q) @ (k * k).T).max(initial=0.0)
        out = p @ v
        return out, 1.01 * half * (np.abs(out) + p @ np.abs(v)) + 2.0 ** -24 * ((16 + 16 * a) * np.abs(v).max() + 2)


def unpack(codes):
    """Two codes a byte, the first in the lower half, along the last dimension."""
    return torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
