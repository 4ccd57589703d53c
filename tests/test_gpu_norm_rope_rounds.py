"""Norm and rotation of prompts whose tokens have more rows than a workgroup
takes at once: its rounds, waves whose rows are of two kinds in a later round,
tokens of more than 64 rows; in place too.  Against the reference of
tests/test_gpu_norm_rope.py, within the bound that is derived there."""
import pytest
import torch

import paper_2607_00760_amd as M
from test_gpu_norm_rope import DT, check, reference

pytestmark = pytest.mark.gpu

D = 128
# sequences, tokens, query heads, kv heads, with values: rows 24, 40, 48, 36, 32, 17, 80, 72, 130 a token
SHAPES = [(1, 520, 16, 8, False), (1, 520, 32, 8, False), (1, 520, 32, 8, True), (2, 300, 28, 4, True), (2, 300, 28, 4, False),
          (1, 513, 7, 5, True), (1, 512, 64, 8, True), (1, 512, 64, 8, False), (3, 171, 128, 1, True)]


def inputs(S, n, hq, hkv, dt, rot, seed):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(S, n, hq + 2 * hkv, D, generator=g).to(dt).cuda()
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(dt).cuda() for _ in range(2)]
    pos = torch.randint(0, 1 << 20, (S, n), generator=g, dtype=torch.int32).cuda()
    inv = torch.pow(500000.0, -torch.arange(0, rot, 2).double() / rot).float().cuda()
    return qkv, qkv[:, :, :hq], qkv[:, :, hq: hq + hkv], qkv[:, :, hq + hkv:], w, pos, inv


@pytest.mark.parametrize("dtype,norm,rot", [("bf16", True, 128), ("fp16", True, 48), ("bf16", False, 64)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("S,n,hq,hkv,with_v", SHAPES)
def test_rounds(S, n, hq, hkv, with_v, inter, dtype, norm, rot):
    dt = DT[dtype]
    _, q, k, v, w, pos, inv = inputs(S, n, hq, hkv, dt, rot, hq + n)
    wq, wk = w if norm else (None, None)
    got = M.qk_norm_rope(q, k, pos, inv, wq, wk, eps=1e-5, interleaved=inter, v=v if with_v else None)
    assert len(got) == (3 if with_v else 2)
    if with_v:
        assert torch.equal(got[2], v.transpose(1, 2))
    for name, y, x, weight in (("q", got[0], q, wq), ("k", got[1].transpose(1, 2), k, wk)):
        want, mag = reference(x, pos, inv, weight, 1e-5, inter)
        check(y, want, mag, dt, name)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("S,n,hq,hkv", [(1, 520, 32, 8), (3, 171, 64, 8)])
def test_rounds_in_place(S, n, hq, hkv, inter):
    """Queries onto themselves inside the projection, whose other rows stay."""
    dt = torch.bfloat16
    qkv, q, k, v, w, pos, inv = inputs(S, n, hq, hkv, dt, 128, 1)
    want = M.qk_norm_rope(q, k, pos, inv, *w, interleaved=inter, v=v)
    rest = qkv[:, :, hq:].clone()
    got = M.qk_norm_rope(q, k, pos, inv, *w, interleaved=inter, v=v, q_out=q)
    assert got[0] is q and all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(qkv[:, :, hq:], rest)
    onto = M.qk_norm_rope(want[0], k, pos, inv, *w, interleaved=inter, q_out=torch.empty_like(q), k_out=k.transpose(1, 2))
    assert torch.equal(onto[1], want[1]) and torch.equal(k.transpose(1, 2), want[1])
