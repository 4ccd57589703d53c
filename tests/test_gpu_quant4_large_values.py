"""Several-token attention over the 4-bit KV cache where bf16 values are next to the
type's largest."""
import pytest
import torch

import _quant4 as Q4
from test_gpu_quant4 import fill, make
from test_gpu_quant4_calls import check_attend

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("H,G,n,L", [(1, 4, 40, 1000), (2, 1, 100, 1000), (128, 4, 2, 2048)])
def test_values_next_to_the_largest(H, G, n, L):
    """A token whose weight is 2^7 times the earlier ones' and whose value is
    2^125: each weight times value is at most that."""
    k, v = torch.zeros((1, H, L, D)), torch.zeros((1, H, L, D))
    k[:, :, L // 4 // 64 * 64:, 0] = 5.0                       # (whole blocks: rows of equal keys are exact)
    v[:, :, L // 4 // 64 * 64 + 7, 3] = 2.0 ** 125
    v[..., 5] = 1.0
    k, v = k.bfloat16(), v.bfloat16()
    c = make(1, H, G, "bf16", 64, L)
    fill(c, k, v, [L])
    q = torch.zeros((1, n, H * G, D))
    q[..., 0] = 1.0
    q = q.bfloat16()
    out = c.attend(q.cuda(), 1.0, causal=False)
    assert out.isfinite().all()
    ref = Q4.Pair(k[0, 0], v[0, 0], 64)                        # (every head's)
    check_attend(out[:, :, :G], [[ref]], q[:, :, :G], G, [n], 1.0, causal=False)
    assert (out.view(1, n, H, G, D) == out[:, :, None, :G]).all()
