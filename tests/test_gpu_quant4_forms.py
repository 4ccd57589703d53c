"""Every form of the 4-bit KV cache's launches against a reference: many runs of a
sequence (joined in groups), more pairs than a launch has runs for, more sequences
than a wave has lanes, row tiles that are workgroups of their own, long appends
without room."""
import math

import numpy as np
import pytest
import torch

import _quant4 as Q4
import paper_2607_00760_amd as M
from test_gpu_quant4 import D, DT, SCALE, check_state, fill, make, pairs, queries, tokens
from test_gpu_quant4_calls import check_decode
from test_gpu_quant4_shares import lengths

pytestmark = pytest.mark.gpu


def random_cache(S, H, G, dtype, block, lens, seed):
    """Codes and grids drawn on the GPU, as if appended."""
    c = make(S, H, G, dtype, block, max(lens), dirty=False)
    g = torch.Generator(device="cuda").manual_seed(seed)
    c.k.random_(0, 256, generator=g)
    c.v.random_(0, 256, generator=g)
    for t in (c.k_grid, c.v_grid):
        t[..., 0, :] = (torch.rand(t[..., 0, :].shape, generator=g, device="cuda") * 0.2 + 0.05).to(t.dtype)
        t[..., 1, :] = -7.5 * t[..., 0, :]
    for t in (c.k_tail, c.v_tail):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    c.lens.copy_(torch.tensor(lens, dtype=torch.int32, device="cuda")[:, None].expand(S, H))
    return c


def held(c, s, h, L):
    """What a pair's codes stand for in fp64, and how large the terms of its products are."""
    B = c.params.block
    nb = L // B
    kg, vg = c.k_grid[s, h, :nb].double(), c.v_grid[s, h, :nb].double()
    kc, vc = Q4.unpack(c.k[s, h, :nb]).double(), Q4.unpack(c.v[s, h, :nb]).transpose(1, 2).double()
    kt, vt = c.k_tail[s, h, : L % B].double(), c.v_tail[s, h, :, : L % B].T.double()
    k = torch.cat(((kg[:, 1, None] + kg[:, 0, None] * kc).flatten(0, 1), kt))
    v = torch.cat(((vg[:, 1, :, None] + vg[:, 0, :, None] * vc).flatten(0, 1), vt))
    ka = torch.cat(((kg[:, 1, None].abs() + 31 * kg[:, 0, None] + 0 * kc).flatten(0, 1), kt.abs()))
    va = max((vg[:, 1].abs() + 31 * vg[:, 0]).max().item() if nb else 0.0, vt.abs().max().item() if L % B else 0.0)
    return k, v, ka, va


# runs of a pair: 79 in groups of 16, 157 of 16, 256 of 16, 50 in groups of 8, 500 in groups of 32
@pytest.mark.parametrize("H,n,block", [(1, 20011, 64), (1, 40001, 64), (1, 32773, 32), (4, 25619, 64), (1, 256033, 32)])
@pytest.mark.parametrize("dtype,G", [("bf16", 4), ("fp16", 7), ("fp16", 1), ("bf16", 8)])
def test_runs_joined_in_groups(dtype, G, H, n, block):
    c = random_cache(1, H, G, dtype, block, [n], 100)
    q = queries(1, H * G, DT[dtype], 101).cuda()
    first = c.decode(q, SCALE)
    for _ in range(3):                                         # (the counters are zero again after each call)
        assert torch.equal(c.decode(q, SCALE), first)
    for h in range(H):
        k, v, ka, va = held(c, 0, h, n)
        x = q[0, h * G: (h + 1) * G].double()
        want = torch.softmax(x @ k.T * SCALE, 1) @ v
        a = SCALE * ((x * x) @ (ka * ka).T).max().sqrt().item()
        err = (first[0, h * G: (h + 1) * G].double() - want).abs().max().item()
        assert err <= 2.0 ** -24 * (16 + 16 * a) * va, (h, err)


@pytest.mark.parametrize("S,H,most", [(70, 1, 1500), (300, 1, 700), (130, 3, 400), (65, 8, 300)])
@pytest.mark.parametrize("dtype,block,G", [("bf16", 64, 4), ("fp16", 32, 7)])
def test_many_sequences(dtype, block, G, S, H, most):
    lens = lengths(S, most, S)
    k, v = tokens(S, H, most, DT[dtype], 102)
    c = make(S, H, G, dtype, block, most)
    fill(c, k, v, lens)
    q = queries(S, H * G, DT[dtype], 103)
    out = c.decode(q.cuda(), SCALE)
    assert torch.equal(c.decode(q.cuda(), SCALE), out)
    check_decode(out, pairs(k, v, lens, block), q, G)


# 256 tiles of 256 rows, 256 of 128, 288 of 32: each is one workgroup's
@pytest.mark.parametrize("S,H,G,n,L", [(1, 8, 4, 2048, 3001), (1, 16, 8, 512, 2500), (32, 8, 1, 100, 700), (36, 8, 4, 5, 900)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,block", [("bf16", 64), ("fp16", 32)])
def test_tiles_of_one_workgroup(dtype, block, causal, S, H, G, n, L):
    dt = DT[dtype]
    lens = [max(L - 37 * s, 1) for s in range(S)]
    c = random_cache(S, H, G, dtype, block, lens, 104)
    q = queries(S, H * G, dt, 105, n).cuda()
    m = [n if s % 3 != 1 else n // 2 for s in range(S)]
    out = c.attend(q, SCALE, torch.tensor(m, dtype=torch.int32, device="cuda"), causal=causal)
    k, v = c.read(L)
    half = torch.finfo(dt).eps / 2
    for s in range(S):
        assert not out[s, m[s]:].any()
        for h in range(H):
            kk, vv = k[s, h, : lens[s]].double(), v[s, h, : lens[s]].double()
            x = q[s, : m[s], h * G: (h + 1) * G].reshape(-1, D).double()
            z = x @ kk.T * SCALE
            a = SCALE * ((x * x) @ (kk * kk).T).max().sqrt().item()
            if causal:
                last = (lens[s] - m[s] + torch.arange(m[s], device="cuda")).repeat_interleave(G)
                z = z.masked_fill(torch.arange(lens[s], device="cuda") > last[:, None], -math.inf)
            p = torch.softmax(z, 1).nan_to_num(0.0)            # (rows that attend nothing)
            want = p @ vv
            tol = 1.01 * half * (want.abs() + p @ vv.abs()) + 2.0 ** -24 * ((16 + 16 * a) * vv.abs().max().item() + 2)
            err = (out[s, : m[s], h * G: (h + 1) * G].reshape(-1, D).double() - want).abs()
            assert (err <= tol).all(), (s, h, err.max().item())


@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_long_appends_without_room(dtype, block):
    """More blocks than a call's workgroups count: a sequence that lacks room by one
    token keeps what it had, the others take theirs."""
    n, H, had = 37 * block + 9, 2, [0, 40, 41, 0, 5]
    cap = n + 40
    cap = -(-cap // block) * block
    had[2] = cap - n + 1
    S = len(had)
    k, v = tokens(S, H, had[2] + n, DT[dtype], 106)
    c = make(S, H, 4, dtype, block, cap)
    fill(c, k, v, had)
    take = [n, n, n, 0, n]
    kc, vc = (torch.stack([x[s, :, had[s]: had[s] + n] for s in range(S)]).cuda() for x in (k, v))
    before = {name: t[2].clone() for name, t in c.tensors().items()}
    c.append(kc, vc, torch.tensor(take, dtype=torch.int32, device="cuda"))
    assert c.refused.tolist() == [0, 0, 1, 0, 0]
    lens = [a + b if a + b <= cap else a for a, b in zip(had, take)]
    check_state(c, pairs(k, v, lens, block), lens)
    for name, t in c.tensors().items():
        assert torch.equal(t[2].view(torch.uint8), before[name].view(torch.uint8)), name


def test_a_batch_is_its_sequences():
    """Each sequence of a ragged batch as it would be alone: both sides are within
    the reference's bound of each output."""
    lens, H, G, n = [1100, 3, 640, 64], 2, 4, 70
    k, v = tokens(4, H, 1100, torch.bfloat16, 107)
    c = make(4, H, G, "bf16", 64, 1100)
    fill(c, k, v, lens)
    q = queries(4, H * G, torch.bfloat16, 108, n)
    out = c.attend(q.cuda(), SCALE).cpu().double().numpy()
    for s, L in enumerate(lens):
        one = make(1, H, G, "bf16", 64, 1100)
        fill(one, k[s:s + 1], v[s:s + 1], [L])
        alone = one.attend(q[s:s + 1].cuda(), SCALE)[0].cpu().double().numpy()
        for h in range(H):
            p = Q4.Pair(k[s, h, :L], v[s, h, :L], 64)
            x = q[s, :, h * G: (h + 1) * G].reshape(-1, D).float().numpy()
            _, tol = p.attend(x, SCALE, np.repeat(L - n + np.arange(n), G))
            err = np.abs(out[s, :, h * G: (h + 1) * G] - alone[:, h * G: (h + 1) * G]).reshape(-1, D)
            assert (err <= 2 * tol).all(), (s, h, err.max())
