"""The forms of the block selection that only large caches take: scoring runs of
several units, and pairs of so many blocks that a thread reads its scores again
in every pass.  The lists of the blocks taken are compared with a reference in
64 bits (whole numbers until the last products, which are fp32's)."""
import math

import numpy as np
import pytest
import torch

import _quant as R
import paper_2607_00760_amd as M

pytestmark = pytest.mark.gpu

D = 128
SCALE = 1.0 / math.sqrt(D)


def over(a, x):
    return torch.full_like(x, a) / x


def scores(k, q, B):
    """fp32 scores of the whole blocks of k [n][D] for the group q [G][D], on the GPU."""
    nb = k.shape[0] // B
    x = k[: nb * B].view(nb, B, D)
    top, low = x.amax(1).float(), x.amin(1).float()
    a = torch.maximum(top.abs(), low.abs()).amax(1).clamp_min(2.0 ** -100)
    unit = over(127.0, a)[:, None]
    hi, lo = (top * unit).ceil().clamp(-127, 127).double(), (low * unit).floor().clamp(-127, 127).double()
    aq = q.float().abs().amax(1).clamp_min(2.0 ** -100)
    q8 = (q.float() * over(127.0, aq)[:, None]).round().double()
    whole = hi @ q8.clamp_min(0).T.contiguous() + lo @ q8.clamp_max(0).T.contiguous()
    return (whole.float() * (aq / torch.full_like(aq, 127.0))).amax(1) * (a / torch.full_like(a, 127.0))


def taken(sc, num, den):
    """Ascending list of the blocks taken: score descending, index ascending."""
    nb = sc.numel()
    want = min(nb, max(1, -(-nb * num // den)))
    return torch.sort(sc, descending=True, stable=True).indices[:want].sort().values.int()


def attended(k, v, q, picked, B):
    """[G][D] fp64 over the blocks `picked` and the tail, and the largest |logit|."""
    rows = torch.cat([torch.arange(b * B, (b + 1) * B) for b in picked.tolist()] + [torch.arange(k.shape[0] // B * B, k.shape[0])])
    r = R.Pair(k.cpu()[rows], v.cpu()[rows], "e4m3", B)
    return r.attend(q.float().cpu().numpy(), SCALE)


def run(lens, H, B, cap, share, compare, ties=()):
    S, G, dt = len(lens), 3, torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(S + H)
    k = torch.empty(S, H, max(lens), D, dtype=dt, device="cuda")
    for s in range(S):
        k[s] = torch.randn(H, max(lens), D, generator=g, device="cuda").to(dt)
    for s, h, a, b, step in ties:                              # blocks a, a + step, .. < b are the same
        for at in range(a + step, b, step):
            k[s, h, at * B: (at + 1) * B] = k[s, h, a * B: (a + 1) * B]
    q = torch.randn(S, H * G, D, generator=g, device="cuda").to(dt)
    c = M.QuantCache(M.QuantParams(H, G, "bf16", "e4m3", B), S, cap)
    lens_dev = torch.tensor(lens, dtype=torch.int32, device="cuda")
    c.append(k, k, lens_dev)
    blocks = torch.empty_like(c.k_scale, dtype=torch.int32)
    for _ in range(2):
        blocks.fill_(77)
        out = c.decode_selected(q, SCALE, share, blocks=blocks)
        for s, h in compare:
            x, qs = k[s, h, : lens[s]], q[s, h * G: (h + 1) * G]
            want = taken(scores(x, qs, B), *share)
            assert torch.equal(blocks[s, h, : want.numel()], want), (s, h)
            assert (blocks[s, h, want.numel():] == -1).all(), (s, h)
    for s, h in compare[:3]:
        x, qs = k[s, h, : lens[s]], q[s, h * G: (h + 1) * G]
        o, zmax = attended(x, x, qs, taken(scores(x, qs, B), *share), B)
        got = out[s, h * G: (h + 1) * G].double().cpu().numpy()
        assert np.linalg.norm(got - o) / np.linalg.norm(o) < R.bound(zmax), (s, h)


@pytest.mark.parametrize("S,H", [(30, 2), (30, 4), (20, 8)])
def test_scoring_runs_of_several_units(S, H):
    """More than 1024 units of 64 blocks: runs of 2, 3 and 3 units, whose last
    ones are of any length down to a block."""
    lens = [(1025 + 37 * s % 300) * 32 + s % 32 for s in range(S)]
    lens[3], lens[4], lens[5], lens[S - 1] = 0, 5, 1088 * 32, 1089 * 32
    assert sum(-(-(n // 32) // 64) for n in lens) * H > 1024 and max(lens) // 32 > 1024
    run(lens, H, 32, max(lens), (1, 12), [(0, 0), (5, H - 1), (S - 1, 1), (2, 0), (3, 0), (4, 1), (S - 2, H - 1)], ties=((2, 0, 10, 900, 3),))


@pytest.mark.parametrize("nb", [1025, 5003, 33001])
def test_scores_read_again(nb):
    """Room for more than 32768 blocks a pair, and more scores than threads: from
    two a thread to 33, equal ones among them, on either side of the threshold."""
    run([nb * 32 + 7, nb // 3 * 32], 1, 32, 32770 * 32 + 40000, (1, 40), [(0, 0), (1, 0)], ties=((0, 0, 4, nb, 7), (1, 0, 0, nb // 3, 2)))


def test_registers_of_keys():
    """Room for up to 16384 and 32768 blocks: every thread's keys in use."""
    for nb in (16300, 32600):
        run([nb * 32 + 1], 1, 32, nb * 32 + 1, (1, 64), [(0, 0)], ties=((0, 0, 1, nb, 11),))
