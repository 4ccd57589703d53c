"""Sums of several-token attention over the 4-bit KV cache where they could lose:
a token that has nearly all weight before or after a million small ones, down to
the least weights of fp16."""
import math

import numpy as np
import pytest
import torch

import paper_2607_00760_amd as M
from test_gpu_quant4 import DT

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("dtype,n,power", [("fp16", 1 << 20, 20.0), ("fp16", 1 << 20, 25.2), ("fp16", 1 << 20, 26.0), ("fp16", 1 << 20, 28.0),
                                           ("fp16", 1 << 20, 31.0), ("bf16", 1 << 21, 25.2), ("bf16", 1 << 21, 22.0)])
def test_a_dominating_token(dtype, n, power, first):
    """One token's weight is 2^power times that of each other one, and its values
    are zeros: the output is the others' share, R / (1 + R), R = (n - 1) / 2^power.
    (256 row tiles: a workgroup walks every token.)"""
    H, G, m, dt = 8, 4, 2048, DT[dtype]
    c = M.Quant4Cache(M.Quant4Params(H, G, dtype, 64), 1, n)
    at = 0 if first else n - 1
    k = torch.zeros((1, H, n, D), dtype=dt, device="cuda")
    v = torch.full((1, H, n, D), -1.0, dtype=dt, device="cuda")
    k[:, :, at, 0] = 4.0
    v[:, :, at] = 0.0
    c.append(k, v)
    del k, v
    kept = c.read(64, 0 if first else n - 64)[0][0, :, 0 if first else 63, 0].double().cpu().numpy()
    q = torch.zeros((1, m, H * G, D), dtype=dt, device="cuda")
    q[..., 0] = 8.0
    scale = float(np.float32(power * math.log(2.0) / (8.0 * kept[0])))
    out = c.attend(q, scale, causal=False).double()
    w = math.exp(-8.0 * kept[0] * scale)
    want = -(n - 1) * w / (1.0 + (n - 1) * w)
    half = torch.finfo(dt).eps / 2
    # relative: the output's rounding and a weight's, half a step each; of fp16 weights
    # also half of 2^-24 next to 2^10 times the weight; fp32 sums of n / 16 matrix
    # products and of n / 64 steps, and 2^-18 of the logits'
    tol = 1.01 * 2 * half + (2.0 ** (power - 35) if dtype == "fp16" else 0.0) + (n / 16 + n / 64) * 2.0 ** -24 + 2.0 ** -18
    err = (out - want).abs().max().item() / abs(want)
    assert kept.min() == kept.max() and err <= tol, (err, tol)
