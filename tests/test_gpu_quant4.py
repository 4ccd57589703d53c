"""The 4-bit KV cache on the GPU against tests/_quant4.py: what append writes and
read gives, bit for bit, and attention of one and of several query tokens."""
import math

import numpy as np
import pytest
import torch

import _quant as Q8
import _quant4 as Q4
import paper_2607_00760_amd as M

pytestmark = pytest.mark.gpu
D = 128
SCALE = 1 / math.sqrt(D)
DT = {"fp16": torch.float16, "bf16": torch.bfloat16}


def tokens(S, H, n, dt, seed, strong=4.0):
    """K and V [S][H][n][D] on the CPU; some channels of K strong and off zero."""
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn((S, H, n, D), generator=g) for _ in range(2))
    k[..., 3::37] = k[..., 3::37] * strong + 2 * strong
    return k.to(dt), v.to(dt)


def make(S, H, G, dtype, block, cap, dirty=True):
    c = M.Quant4Cache(M.Quant4Params(num_kv_heads=H, group_size=G, dtype=dtype, block=block), S, cap)
    if dirty:                                                  # what is not a token's takes part in nothing
        for n in ("k", "v"):
            getattr(c, n).fill_(0x5a)
        for n in ("k_grid", "v_grid", "k_tail", "v_tail"):
            getattr(c, n).fill_(float("nan"))
    return c


def fill(c, k, v, lens, cuts=1):
    """Each sequence's first lens[s] tokens, in `cuts` parts."""
    done = [0] * len(lens)
    for i in range(cuts):
        to = [L * (i + 1) // cuts for L in lens]
        m = max(max(b - a for a, b in zip(done, to)), 1)
        kc, vc = (torch.full((x.shape[0], x.shape[1], m, D), float("nan"), dtype=x.dtype) for x in (k, v))
        for s, (a, b) in enumerate(zip(done, to)):
            kc[s, :, : b - a], vc[s, :, : b - a] = k[s, :, a:b], v[s, :, a:b]
        c.append(kc.cuda(), vc.cuda(), torch.tensor([b - a for a, b in zip(done, to)], dtype=torch.int32, device="cuda"))
        done = to


def pairs(k, v, lens, block):
    return [[Q4.Pair(k[s, h, :L], v[s, h, :L], block) for h in range(k.shape[1])] for s, L in enumerate(lens)]


def check_state(c, ref, lens):
    got = {n: t.cpu() for n, t in c.tensors().items()}
    B = c.params.block
    assert got["lens"].tolist() == [[L] * c.params.num_kv_heads for L in lens]
    for s, L in enumerate(lens):
        for h, p in enumerate(ref[s]):
            nb, rest = L // B, L % B
            for b in range(nb):
                (kc, ks, kz), (vc, vs, vz) = p.kc[b], p.vc[b]
                assert np.array_equal(Q4.unpack(got["k"][s, h, b]).numpy(), kc.T), (s, h, b)
                assert np.array_equal(Q4.unpack(got["v"][s, h, b]).numpy(), vc.T), (s, h, b)
                assert np.array_equal(got["k_grid"][s, h, b].float().numpy(), np.stack((ks, kz)))
                assert np.array_equal(got["v_grid"][s, h, b].float().numpy(), np.stack((vs, vz)))
            assert np.array_equal(got["k_tail"][s, h, :rest].float().numpy(), p.k[nb * B:])
            assert np.array_equal(got["v_tail"][s, h, :, :rest].float().numpy(), p.v[nb * B:].T)
            assert (got["k"][s, h, nb:] == 0x5a).all() and (got["v"][s, h, nb:] == 0x5a).all()
            assert got["k_grid"][s, h, nb:].isnan().all() and got["v_grid"][s, h, nb:].isnan().all()


LENS = {32: [0, 1, 31, 32, 33, 64, 97, 300], 64: [0, 1, 63, 64, 65, 128, 200, 577]}


@pytest.mark.parametrize("cuts", [1, 3])
@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_append(dtype, block, cuts):
    lens = LENS[block]
    k, v = tokens(len(lens), 2, max(lens), DT[dtype], 1)
    c = make(len(lens), 2, 4, dtype, block, max(lens) + 70)
    fill(c, k, v, lens, cuts)
    check_state(c, pairs(k, v, lens, block), lens)
    assert c.refused.tolist() == [0] * len(lens)


@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_token_by_token_is_the_same(dtype, block):
    n = 2 * block + 5
    k, v = tokens(2, 3, n, DT[dtype], 2)
    c = make(2, 3, 2, dtype, block, n)
    kd, vd = k.cuda(), v.cuda()
    for t in range(n):
        c.append(kd[:, :, t], vd[:, :, t])
    check_state(c, pairs(k, v, [n, n], block), [n, n])


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_rows_of_every_kind(dtype):
    """Constant rows, zeros, tiny, subnormal and huge ones, and the type's range."""
    dt, B = DT[dtype], 32
    big, tiny = torch.finfo(dt).max, torch.finfo(dt).tiny
    x = torch.randn((1, 1, 3 * B, D), generator=torch.Generator().manual_seed(3))
    x[..., 0], x[..., 1] = 0.0, 5.0
    x[..., 2] = torch.linspace(-1, 1, 3 * B) * big
    x[..., 3] = x[..., 3].sign() * big
    x[..., 4] *= tiny
    x[..., 5] *= tiny / 64
    x[0, 0, 1], x[0, 0, 2] = 0.0, -big
    x[0, 0, 3] = x[0, 0, 3] * tiny / 16
    x = x.clamp(-big, big).to(dt)
    c = make(1, 1, 1, dtype, B, 3 * B)
    c.append(x.cuda(), x.flip(3).cuda())
    ref = pairs(x, x.flip(3), [3 * B], B)
    check_state(c, ref, [3 * B])
    k, v = c.read(3 * B)
    for got, want in zip((k, v), ref[0][0].read()):
        assert torch.equal(got[0, 0].cpu(), want) and torch.isfinite(want).all()


@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_read(dtype, block):
    lens = LENS[block]
    S, H, n = len(lens), 2, 150
    k, v = tokens(S, H, max(lens), DT[dtype], 4)
    c = make(S, H, 4, dtype, block, max(lens) + 70)
    fill(c, k, v, lens)
    ref = pairs(k, v, lens, block)
    starts = [0, 0, -5, 3, 33, 63, -200, lens[7] - 140]
    out = torch.full((S, n, 2, H, D + 8), 7.0, dtype=DT[dtype], device="cuda")[..., :D]       # rows of any strides
    ko, vo = out[:, :, 0].transpose(1, 2), out[:, :, 1].transpose(1, 2)
    got = c.read(n, torch.tensor(starts, dtype=torch.int32, device="cuda"), ko, vo)
    assert got[0] is ko and got[1] is vo
    for s, L in enumerate(lens):
        a, b = max(starts[s], 0), max(min(starts[s] + n, L), 0)
        for h in range(H):
            for have, want in zip((ko, vo), ref[s][h].read()):
                have = have[s, h].cpu()
                held = torch.zeros(n, dtype=torch.bool)
                if a < b:
                    held[a - starts[s]: b - starts[s]] = True
                    assert torch.equal(have[held], want[a:b])
                assert (have[~held] == 7.0).all()
    k2, v2 = c.read(n, 3)                                      # new tensors: zeros where nothing is held
    for s, L in enumerate(lens):
        m = max(0, min(n, L - 3))
        assert torch.equal(k2[s, 1, :m].cpu(), ref[s][1].read()[0][3: 3 + m]) and (k2[s, :, m:] == 0).all() and (v2[s, :, m:] == 0).all()
    assert c.read(0)[0].shape == (S, H, 0, D)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_read_of_the_8_bit_cache(dtype, block, fmt):
    lens = LENS[block]
    S, H, n = len(lens), 2, max(lens) + 9
    k, v = tokens(S, H, max(lens), DT[dtype], 5)
    c = M.QuantCache(M.QuantParams(num_kv_heads=H, group_size=4, dtype=dtype, format=fmt, block=block), S, max(lens))
    fill(c, k, v, lens)
    ko, vo = (torch.full((S, H, n, D), 7.0, dtype=DT[dtype], device="cuda") for _ in range(2))
    c.read(n, -2, ko, vo)
    for s, L in enumerate(lens):
        for h in range(H):
            p = Q8.Pair(k[s, h, :L], v[s, h, :L], fmt, block)
            for have, codes, raw in ((ko, p.kc, p.k), (vo, p.vc, p.v)):
                want = [c.astype(np.float32) * a for c, a in codes] + [raw[p.nb * block:]]
                want = torch.from_numpy(np.concatenate(want)).to(DT[dtype])
                have = have[s, h].cpu()
                assert torch.equal(have[2: 2 + L], want) and (have[:2] == 7.0).all() and (have[2 + L:] == 7.0).all()


def queries(S, Hq, dt, seed, n=None):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((S, Hq, D) if n is None else (S, n, Hq, D), generator=g).to(dt)


@pytest.mark.parametrize("G", [1, 3, 4, 5, 7, 8])
@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_decode(dtype, block, G):
    lens = LENS[block] + [2500]
    S, H, dt = len(lens), 2, DT[dtype]
    k, v = tokens(S, H, max(lens), dt, 6 + G)
    c = make(S, H, G, dtype, block, max(lens) + 1)
    fill(c, k, v, lens)
    q = queries(S, H * G, dt, 7 + G)
    out = c.decode(q.cuda(), SCALE).cpu().double().numpy()
    worst = 0.0
    for s, row in enumerate(pairs(k, v, lens, block)):
        for h, p in enumerate(row):
            want, tol = p.decode(q[s, h * G: (h + 1) * G].float().numpy(), SCALE)
            err = np.abs(out[s, h * G: (h + 1) * G] - want).max()
            worst = max(worst, err / tol if tol else err)
            assert err <= tol, (s, h, err, tol)
    print(f"largest share of the bound: {worst:.3f}")


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [1, 5, 8, 9, 40, 130])
@pytest.mark.parametrize("G,block,dtype", [(4, 64, "bf16"), (4, 32, "fp16"), (1, 64, "fp16"), (7, 32, "bf16"), (8, 64, "fp16"), (3, 64, "bf16")])
def test_attend(dtype, block, G, n, causal):
    lens = LENS[block] + [1500]
    S, H, dt = len(lens), 2, DT[dtype]
    k, v = tokens(S, H, max(lens), dt, 16 + G)
    c = make(S, H, G, dtype, block, max(lens) + 1)
    fill(c, k, v, lens)
    m = [n, n, max(0, n - 1), n, (n + 1) // 2, 0, n, n, n]     # (more queries than tokens where a sequence is short)
    q = queries(S, H * G, dt, 17 + G, n)
    qd = torch.full((S, n, H * G + 1, D), float("nan"), dtype=dt, device="cuda")[:, :, 1:]    # rows of any strides
    for s in range(S):
        qd[s, : m[s]] = q[s, : m[s]].cuda()
    out = torch.full((S, H * G, n, D), 7.0, dtype=dt, device="cuda").transpose(1, 2)
    assert c.attend(qd, SCALE, torch.tensor(m, dtype=torch.int32, device="cuda"), causal=causal, out=out) is out
    got = out.cpu().double().numpy()
    worst = 0.0
    for s, (L, row) in enumerate(zip(lens, pairs(k, v, lens, block))):
        assert (got[s, m[s]:] == 7.0).all()
        last = np.repeat(L - m[s] + np.arange(m[s]) if causal else np.full(m[s], L - 1), G)
        for h, p in enumerate(row):
            x = q[s, : m[s], h * G: (h + 1) * G].reshape(-1, D).float().numpy()
            want, tol = p.attend(x, SCALE, last)
            err = np.abs(got[s, : m[s], h * G: (h + 1) * G].reshape(-1, D) - want)
            assert (err <= tol).all(), (s, h, err.max())
            worst = max(worst, (err / np.maximum(tol, 1e-30)).max(initial=0.0))
    print(f"largest share of the bound: {worst:.3f}")
