"""Attention over the 8-bit cache for every finite value that the types hold:
value scales far apart, with the softmax's weight on any of them; values next
to the type's largest; queries of very different channels; and values that are
not finite, wherever they stand.  Against tests/_quant.py, within the error
that the arithmetic allows (_quant.bound)."""
import math

import numpy as np
import pytest
import torch

import _quant as R
import paper_2607_00760_amd as M

pytestmark = pytest.mark.gpu

D = 128
SCALE = 1.0 / math.sqrt(D)
DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
FORMS = [(f, d, b) for f in ("e4m3", "int8") for d in ("fp16", "bf16") for b in (32, 64)]


def make(fmt, dtype, block, S, H, G, cap):
    """A cache whose unwritten parts are NaN."""
    c = M.QuantCache(M.QuantParams(H, G, dtype, fmt, block), S, cap)
    for n in c.TENSORS:
        if n != "lens":
            getattr(c, n).view(torch.uint8).fill_(0xff)
    return c


def check(c, k, v, q, G, where):
    """k, v [H][n][D], q [H * G][D] of one sequence: every head for itself."""
    c.append(k[None].cuda(), v[None].cuda())
    out, part = c.decode(q[None].cuda(), SCALE)[0], c.decode_selected(q[None].cuda(), SCALE, (2, 3))[0]
    p = c.params
    for h in range(k.shape[0]):
        r = R.Pair(k[h], v[h], p.format, p.block)
        at = slice(h * G, (h + 1) * G)
        for got, picked, name in ((out, None, "all"), (part, r.select(q[at].float().numpy(), 2, 3), "selected")):
            for g in range(G):
                qs = q[h * G + g][None].float().numpy()
                want, zmax = r.attend(qs, SCALE, picked)
                x = got[h * G + g].double().cpu().numpy()
                assert np.isfinite(x).all(), f"{where} {name} head {g}"
                rel = np.linalg.norm(x - want[0]) / np.linalg.norm(want)
                assert rel < R.bound(zmax), f"{where} {name} head {g}: rel {rel:.2e} of {R.bound(zmax):.2e}"


def apart(fmt, dtype, block, bits, nb, tail, big):
    """Blocks of values about 2^`bits` apart; big(b): whether block b (nb: the
    unfinished one) is a large one.  Keys of large blocks lie against a sign
    vector, the others along it: the heads put their weight on the small blocks,
    on the large ones, on both alike, and where the two products are alike."""
    B, G, dt = block, 4, DT[dtype]
    g = torch.Generator().manual_seed(bits + nb)
    n = nb * B + tail
    u = torch.sign(torch.randn(D, generator=g))
    is_big = torch.tensor([big(i // B) for i in range(n)])
    top = min(13, bits // 2) if dtype == "fp16" else bits // 2
    v = torch.randn(n, D, generator=g)
    v = (v * torch.where(is_big, 2.0 ** top, 2.0 ** (top - bits))[:, None]).to(dt)
    k = (u * torch.where(is_big, -1.0, 1.0)[:, None] + 0.05 * torch.randn(n, D, generator=g)).to(dt)
    # z = +-SCALE * D * a; the large blocks' weight is exp(-2 z)
    unit = math.log(2.0) / (2 * SCALE * D)
    a = torch.tensor([min(bits + 30.0, 120.0) * unit, -20.0 * unit, 0.0, min(bits, 60.0) * unit])
    q = (a[:, None] * u + 0.02 * torch.randn(G, D, generator=g)).to(dt)
    check(make(fmt, dtype, B, 1, 1, G, n), k[None], v[None], q, G, f"{bits} bits, {nb} blocks + {tail}")


@pytest.mark.parametrize("fmt,dtype,block", FORMS)
def test_value_scales_apart(fmt, dtype, block):
    """A wave meets large blocks before small ones and the other way round; runs
    of large blocks are joined with runs of small ones."""
    for bits in (20, 28, 30) if dtype == "fp16" else (24, 32, 40, 90, 200):
        for nb, big in ((9, lambda b: b < 4), (9, lambda b: b >= 5), (40, lambda b: b % 8 < 4), (70, lambda b: b < 40)):
            apart(fmt, dtype, block, bits, nb, 0, big)


@pytest.mark.parametrize("fmt,dtype,block", FORMS)
def test_unfinished_block_apart(fmt, dtype, block):
    """The unfinished block's values far above or below the whole blocks', or alone."""
    for bits in (20, 30) if dtype == "fp16" else (40, 100, 200, 240):
        for nb in (0, 1, 8, 40):
            apart(fmt, dtype, block, bits, nb, 7, lambda b: b == nb)
            apart(fmt, dtype, block, bits, nb, block - 1, lambda b: b < nb)


@pytest.mark.parametrize("fmt,dtype,block", FORMS)
def test_unfinished_block_of_mixed_values(fmt, dtype, block):
    """Tokens of the unfinished block of very different magnitudes, the weight
    on the small ones, on the large ones, or where the products are alike."""
    dt, G = DT[dtype], 3
    g = torch.Generator().manual_seed(23)
    bits = 20 if dtype == "fp16" else 100
    top = 14 if dtype == "fp16" else 50
    for n in (block - 1, 2 * block + 9):
        u = torch.sign(torch.randn(D, generator=g))
        large = torch.arange(n) % 3 == 0
        v = (torch.randn(n, D, generator=g) * torch.where(large, 2.0 ** (top - 2), 2.0 ** (top - bits))[:, None]).to(dt)
        if n > block:
            v[: n // block * block] = torch.randn(n // block * block, D, generator=g).to(dt)
        k = (u * torch.where(large, -1.0, 1.0)[:, None] + 0.05 * torch.randn(n, D, generator=g)).to(dt)
        unit = math.log(2.0) / (2 * SCALE * D)
        a = torch.tensor([min(bits + 30.0, 120.0) * unit, -20.0 * unit, min(bits, 60.0) * unit])
        q = (a[:, None] * u + 0.02 * torch.randn(G, D, generator=g)).to(dt)
        check(make(fmt, dtype, block, 1, 1, G, n), k[None], v[None], q, G, f"{n} tokens")


@pytest.mark.parametrize("fmt,dtype,block", FORMS)
@pytest.mark.parametrize("G", [2, 4, 7])
def test_weights_on_zeros(fmt, dtype, block, G):
    """The softmax's weight lies on tokens whose values, or codes, are zeros: the
    output is what the others bring, 2^20 to 2^110 below their values."""
    dt = DT[dtype]
    g = torch.Generator().manual_seed(G)
    u = torch.sign(torch.randn(D, generator=g))
    unit = math.log(2.0) / (2 * SCALE * D)
    a = torch.tensor([20.0, 35.0, 50.0, 65.0, 80.0, 95.0, 110.0][-G:]) * unit
    q = (a[:, None] * u).to(dt)
    for n in (block - 5, 2 * block, 41 * block + 17):
        none = torch.rand(n, generator=g) < 0.3
        none[0], none[-1] = True, False
        for small in (0.0, 2.0 ** -20):                        # (codes of zero next to the block's others)
            v = torch.randn(n, D, generator=g) * torch.where(none, small, 1.0)[:, None]
            if small and n % block:
                v[none & (torch.arange(n) >= n // block * block)] = 0.0
            k = u * torch.where(none, 1.0, -1.0)[:, None]
            check(make(fmt, dtype, block, 1, 1, G, n), k.to(dt)[None], v.to(dt)[None], q, G, f"{n} tokens, {small}")


@pytest.mark.parametrize("fmt,dtype,block", FORMS)
@pytest.mark.parametrize("nb,tail", [(0, 1), (0, 5), (1, 0), (9, 31), (70, 3), (700, 1)])
def test_values_next_to_the_largest(fmt, dtype, block, nb, tail):
    """Channels of one sign at the type's largest: an average of them is finite
    however many tokens there are, in the unfinished block as in whole ones."""
    dt, G, n = DT[dtype], 4, nb * block + tail
    g = torch.Generator().manual_seed(nb)
    top = torch.finfo(dt).max
    v = torch.full((n, D), top)
    v[:, 1::2] *= torch.sign(torch.randn(n, D // 2, generator=g))
    v[:, ::4] *= -1.0
    v = v.to(dt)
    k, q = torch.randn(n, D, generator=g).to(dt), (0.1 * torch.randn(G, D, generator=g)).to(dt)
    check(make(fmt, dtype, block, 1, 1, G, n), k[None], v[None], q, G, f"{n} tokens")


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("bits", [18, 24, 30, 60, 100])
def test_queries_of_far_channels(fmt, block, bits):
    """A bf16 query whose largest channel meets keys of zero: the others, 2^`bits`
    below it, make the logits."""
    G, n = 3, 9 * block + 5
    g = torch.Generator().manual_seed(bits)
    k, v = torch.randn(n, D, generator=g), torch.randn(n, D, generator=g)
    k[:, 7] = 0.0
    q = torch.randn(G, D, generator=g)
    q[:, 7] = 2.0 ** bits
    q[1] *= 2.0 ** -3
    check(make(fmt, "bf16", block, 1, 1, G, n), k.bfloat16()[None], v.bfloat16()[None], q.bfloat16(), G, f"{bits} bits")


@pytest.mark.parametrize("fmt,dtype,block", FORMS)
def test_values_that_are_not_finite_in_first_blocks(fmt, dtype, block):
    """A NaN or an infinity in a block that a wave meets first, or in the only
    one, shows in its (sequence, kv head) and nowhere else."""
    B, H, G, dt = block, 2, 3, DT[dtype]
    lens = [20 * B + 7, 20 * B + 7, B, 8 * B, 4 * B + 1, 3]
    at = [0, 3 * B + 5, B - 1, 7 * B, 2 * B, 1]                # tokens that are spoilt, of head 1
    S, n = len(lens), max(lens)
    g = torch.Generator().manual_seed(16)
    k, v = (torch.randn(S, H, n, D, generator=g).to(dt) for _ in range(2))
    q = torch.randn(S, H * G, D, generator=g).to(dt)
    lens_dev = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def outputs(kk, vv):
        c = make(fmt, dtype, B, S, H, G, n)
        c.append(kk.cuda(), vv.cuda(), lens_dev)
        return c.decode(q.cuda(), SCALE), c.decode_selected(q.cuda(), SCALE, (1, 1))
    clean = outputs(k, v)
    for bad in (float("nan"), float("inf"), -float("inf")):
        for which in range(2):
            x = [k.clone(), v.clone()]
            for s in range(S):
                x[which][s, 1, at[s], 9] = bad
            for a, b in zip(clean, outputs(*x)):
                a, b = a.view(S, H, G, D), b.view(S, H, G, D)
                assert torch.isfinite(a).all() and torch.equal(a[:, 0], b[:, 0]), (bad, which)
                for s in range(S):
                    if which == 0 and math.isinf(bad) and at[s] >= lens[s] // B * B:
                        continue                               # (a logit of minus infinity is a weight of zero)
                    for h in range(G):
                        assert not torch.isfinite(b[s, 1, h]).all(), (bad, which, s, h)
