"""Norms of rows of any finite magnitude: squares that pass fp32's range on
either side, weights and all.  Against the reference of
tests/test_gpu_norm_rope.py, within the bound that is derived there; where a
result is below bf16's normal range a step is absolute, 2^-133."""
import pytest
import torch

import paper_2607_00760_amd as M
from test_gpu_norm_rope import reference

pytestmark = pytest.mark.gpu

D = 128


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("rot", [64, 128])
@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-12, 1e-6])
def test_rows_of_any_magnitude(inter, rot, eps):
    """bf16 rows from 2^-125 to 2^126, one magnitude each, and rows whose
    channels spread over all of them; the others of the wave are ordinary."""
    S, n, hq, hkv = 1, 5, 13, 3
    g = torch.Generator().manual_seed(rot)
    x = torch.randn(S, n, hq + hkv, D, generator=g)
    at = torch.tensor([-125, -100, -75, -70, -64, -60, -50, -45, 0, 40, 50, 58, 62, 64, 70, 100])
    x[0, :4] *= torch.exp2(at.double())[None, :, None].float()
    x[0, 1] *= 2.0 ** -1
    x[0, 2] *= 2.0 ** 1
    x[0, 3] = x[0, 3].sign() * torch.exp2(torch.randint(-125, 127, (hq + hkv, D), generator=g).float())
    x[0, 0, 15] *= 2.0 ** 24
    x = x.bfloat16()
    assert torch.isfinite(x).all()
    w = [(1 + 0.3 * torch.randn(D, generator=g)).bfloat16().cuda() for _ in range(2)]
    pos = torch.randint(0, 1 << 20, (S, n), generator=g).cuda()
    inv = torch.pow(500000.0, -torch.arange(0, rot, 2).double() / rot).float().cuda()
    q, k = x[:, :, :hq].cuda(), x[:, :, hq:].cuda()
    qo, ko = M.qk_norm_rope(q, k, pos, inv, *w, eps=eps, interleaved=inter)
    for name, y, r, weight in (("q", qo, q, w[0]), ("k", ko.transpose(1, 2), k, w[1])):
        assert torch.isfinite(y).all(), name
        # eps as the call has it, in 32 bits
        want, mag = reference(r, pos, inv, weight, float(torch.tensor(eps, dtype=torch.float32)), inter)
        tol = torch.finfo(torch.bfloat16).eps / 2 * want.abs() + 2.0 ** -20 * mag + 2.0 ** -134
        off = (y.double().cpu() - want).abs()
        assert (off <= tol).all(), f"{name}: {float((off / tol).max()):.2f} of the bound"


def test_rows_of_zeros():
    """Zeros stay zeros next to rows of large values."""
    x = torch.zeros(1, 2, 8, D, dtype=torch.bfloat16, device="cuda")
    x[0, 1, ::2] = 2.0 ** 100
    pos, inv, w = torch.ones(1, 2, dtype=torch.int32, device="cuda"), torch.ones(64, device="cuda"), torch.ones(D, dtype=torch.bfloat16, device="cuda")
    q, _ = M.qk_norm_rope(x, x, pos, inv, w, w)
    assert not q[0, 0].any() and not q[0, 1, 1::2].any() and torch.isfinite(q).all() and (q[0, 1, ::2] != 0).any()
