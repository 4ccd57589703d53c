"""Attention of several query tokens over the 4-bit KV cache where the batch is
shared among workgroups: tiles of rows below, at and past the number that is
shared, sequences of any lengths (some empty, some without queries), and the same
launch replayed after the lengths have changed."""
import math

import numpy as np
import pytest
import torch

from test_gpu_quant4 import D, DT, SCALE, fill, make, pairs, queries, tokens

pytestmark = pytest.mark.gpu


def lengths(S, most, seed):
    """Lengths that differ widely: empty, one, short, and a few of `most`."""
    g = np.random.default_rng(seed)
    lens = np.exp(g.uniform(0, math.log(most), S)).astype(int)
    lens[::5] = most
    lens[2::7] = 0
    return lens.tolist()


# pairs times row tiles: 6, 120 and 255 of 32 rows, 256 (each its own workgroup); 63 and 65 of 128; 40 and 190 of 256
@pytest.mark.parametrize("S,H,G,n", [(3, 2, 3, 9), (40, 3, 4, 5), (51, 5, 8, 2), (64, 4, 4, 3), (9, 7, 1, 100), (13, 5, 1, 100),
                                     (5, 2, 7, 140), (19, 2, 4, 300)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,block", [("bf16", 64), ("fp16", 32)])
def test_shares_of_a_batch(dtype, block, causal, S, H, G, n):
    dt = DT[dtype]
    lens = lengths(S, 1100, S)
    half = [L // 2 for L in lens]
    m = [n if s % 3 else (s // 3) % (n + 1) for s in range(S)]
    k, v = tokens(S, H, 1100, dt, 31 + S)
    c = make(S, H, G, dtype, block, 1101)
    fill(c, k, v, half)
    q = queries(S, H * G, dt, 32 + S, n)
    qd, md = q.cuda(), torch.tensor(m, dtype=torch.int32, device="cuda")
    first = c.attend(qd, SCALE, md, causal=causal)
    replayed = torch.zeros_like(qd)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attend(qd, SCALE, md, causal=causal, out=replayed)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, replayed)
    rest = torch.tensor([L - a for L, a in zip(lens, half)], dtype=torch.int32, device="cuda")
    kc, vc = (torch.zeros((S, H, 550, D), dtype=dt) for _ in range(2))
    for s, (a, L) in enumerate(zip(half, lens)):
        kc[s, :, : L - a], vc[s, :, : L - a] = k[s, :, a:L], v[s, :, a:L]
    c.append(kc.cuda(), vc.cuda(), rest)
    out = c.attend(qd, SCALE, md, causal=causal)
    for _ in range(3):
        replayed.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, replayed)
    got = out.cpu().double().numpy()
    for s, (L, row) in enumerate(zip(lens, pairs(k, v, lens, block))):
        assert (got[s, m[s]:] == 0.0).all()
        last = np.repeat(L - m[s] + np.arange(m[s]) if causal else np.full(m[s], L - 1), G)
        for h, p in enumerate(row):
            x = q[s, : m[s], h * G: (h + 1) * G].reshape(-1, D).float().numpy()
            want, tol = p.attend(x, SCALE, last)
            err = np.abs(got[s, : m[s], h * G: (h + 1) * G].reshape(-1, D) - want)
            assert (err <= tol).all(), (s, h, err.max())


def test_a_batch_is_its_sequences():
    """Each sequence of a ragged batch as it would be alone, within two roundings of
    the results (sums are split otherwise, weights stay the same to their own)."""
    lens, H, G, n = [1100, 3, 640, 64], 2, 4, 70
    k, v = tokens(4, H, 1100, torch.bfloat16, 77)
    c = make(4, H, G, "bf16", 64, 1100)
    fill(c, k, v, lens)
    q = queries(4, H * G, torch.bfloat16, 78, n).cuda()
    out = c.attend(q, SCALE)
    for s, L in enumerate(lens):
        one = make(1, H, G, "bf16", 64, 1100)
        fill(one, k[s:s + 1], v[s:s + 1], [L])
        alone = one.attend(q[s:s + 1].contiguous(), SCALE)[0].double()
        # a weight is rounded relative to another maximum (2^-8 of it either way), the result once
        bound = 2.0 * 2.0 ** -8 * float(v[s, :, :L].double().abs().max()) + 2.0 ** -8 * alone.abs()
        assert ((out[s].double() - alone).abs() <= bound).all()
