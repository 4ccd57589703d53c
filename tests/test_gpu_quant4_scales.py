"""Attention over the 4-bit KV cache with softmax scales at the ends of their
range: zero and subnormal ones over very large logits, the largest over zeros."""
import numpy as np
import pytest
import torch

import paper_2607_00760_amd as M
from test_gpu_quant4 import DT, fill, make, pairs, queries, tokens
from test_gpu_quant4_calls import check_attend, check_decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [0.0, -0.0, 2.0 ** -149, 1e-40, -1e-40, 2.0 ** -126, -2.0 ** -126, 2.0 ** -121, 3e-37])
@pytest.mark.parametrize("G,block", [(4, 64), (7, 32)])
def test_small_scales_of_large_logits(G, block, scale):
    """Sums of q and K about 2^123: their powers are far below one, or small."""
    lens = [1, 40, 64, 333, 1500]
    k, v = tokens(5, 2, 1500, torch.bfloat16, 91, 1.0)
    k = (k.float() * 2.0 ** 58).bfloat16()
    c = make(5, 2, G, "bf16", block, 1500)
    fill(c, k, v, lens)
    ref = pairs(k, v, lens, block)
    big = lambda q: (q.float() * 2.0 ** 60).bfloat16()  # noqa: E731
    q = big(queries(5, 2 * G, torch.bfloat16, 92))
    check_decode(c.decode(q.cuda(), scale), ref, q, G, scale)
    for n in (2, 50):
        q = big(queries(5, 2 * G, torch.bfloat16, 93, n))
        check_attend(c.attend(q.cuda(), scale), ref, q, G, [n] * 5, scale)
        check_attend(c.attend(q.cuda(), scale, causal=False), ref, q, G, [n] * 5, scale, causal=False)


@pytest.mark.parametrize("scale", [2.0 ** 127, -2.0 ** 127, 1e38])
@pytest.mark.parametrize("dtype,block,G", [("fp16", 32, 7), ("bf16", 64, 4)])
def test_large_scales_of_zeros(dtype, block, G, scale):
    lens = [1, 40, 64, 333]
    k, v = tokens(4, 2, 333, DT[dtype], 94)
    c = make(4, 2, G, dtype, block, 400)
    fill(c, k, v, lens)
    ref = pairs(k, v, lens, block)
    for n in (None, 2, 50):
        q = torch.zeros_like(queries(4, 2 * G, DT[dtype], 95, n))
        if n is None:
            check_decode(c.decode(q.cuda(), scale), ref, q, G, 1.0)    # (every logit is zero)
        else:
            check_attend(c.attend(q.cuda(), scale), ref, q, G, [n] * 4, 1.0)


def test_large_scales_of_small_queries():
    """q of 2^-110: the same logits as with ordinary ones."""
    lens = [1, 40, 64, 333]
    k, v = tokens(4, 2, 333, torch.bfloat16, 96)
    c = make(4, 2, 4, "bf16", 64, 400)
    fill(c, k, v, lens)
    ref = pairs(k, v, lens, 64)
    scale = 2.0 ** 107
    for n in (None, 2, 50):
        q = (queries(4, 8, torch.bfloat16, 97, n).float() * 2.0 ** -110).bfloat16()
        if n is None:
            check_decode(c.decode(q.cuda(), scale), ref, q, 4, scale)
        else:
            check_attend(c.attend(q.cuda(), scale), ref, q, 4, [n] * 4, scale)


def test_scales_that_are_refused():
    c = make(1, 1, 1, "bf16", 32, 64, dirty=False)
    q = torch.zeros(1, 1, 128, dtype=torch.bfloat16, device="cuda")
    for scale in (float("inf"), -float("inf"), float("nan"), np.nextafter(np.float32(2.0 ** 127), np.float32(np.inf)), -3e38):
        with pytest.raises(M.MosaicError):
            c.decode(q, scale)
        with pytest.raises(M.MosaicError):
            c.attend(q[:, None], scale)
