"""Attention over the 8-bit cache for every value that the types hold."""
import math

import pytest
import torch

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
