"""Calls around the 8-bit cache and the norm-and-rotation pass that a program
may make beside the ordinary ones."""
import numpy as np
import pytest
import torch

import paper_2607_00760_amd as M

pytestmark = pytest.mark.gpu

D = 128


def test_reset_of_a_list_is_captured():
    """Emptying named sequences copies nothing to the device: a graph records
    it, with the appends that follow, and every replay empties them again."""
    S, H, B = 5, 2, 32
    c = M.QuantCache(M.QuantParams(H, 4, "bf16", "e4m3", B), S, 4 * B)
    g = torch.Generator().manual_seed(0)
    x = torch.randn(S, H, 37, D, generator=g).bfloat16().cuda()
    c.append(x, x)
    c.reset([])
    assert c.lens.tolist() == [[37] * H] * S
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.reset([3, 1, 3])
        c.append(x[:, :, :2], x[:, :, :2])
    torch.cuda.current_stream().wait_stream(side)
    assert c.lens.tolist() == [[n] * H for n in (39, 2, 39, 2, 39)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.reset([3, 1, 3])
        c.append(x[:, :, :2], x[:, :, :2])
    for i in range(1, 4):
        graph.replay()
        assert c.lens.tolist() == [[n] * H for n in (39 + 2 * i, 2, 39 + 2 * i, 2, 39 + 2 * i)], i
        assert torch.equal(c.k_tail[1, :, :2], x[1, :, :2])


def test_reset_of_lists_of_all_kinds():
    S, H = 9, 2
    c = M.QuantCache(M.QuantParams(H, 1, "fp16", "int8", 32), S, 32)
    for named in ([0], [8], [0, 8], [2, 1, 3], [0, 1, 2, 4, 5, 7], list(range(9)), (3, 3), range(4, 9), np.array([6, 0]), {5}):
        c.lens.fill_(7)
        c.reset(named)
        assert c.lens.tolist() == [[0 if s in list(named) else 7] * H for s in range(S)], named
    for bad in ([9], [0, -1], [-9, 3], [2, 100]):
        with pytest.raises(ValueError):
            c.reset(bad)


def test_outputs_whose_rows_overlap_are_refused():
    S, n, H = 2, 3, 4
    x = torch.randn(S, n, H, D, device="cuda").half()
    pos, inv = torch.zeros(S, n, dtype=torch.int32, device="cuda"), torch.ones(64, device="cuda")
    one = torch.empty(1, 1, 1, D, dtype=torch.float16, device="cuda")
    for name, shape in (("q_out", (S, n, H, D)), ("k_out", (S, H, n, D)), ("v_out", (S, H, n, D))):
        with pytest.raises(M.MosaicError, match="overlap"):
            M.qk_norm_rope(x, x, pos, inv, v=x, **{name: one.expand(shape)})
    q, k = M.qk_norm_rope(x[:1, :1, :1].expand(S, n, H, D), x, pos, inv)      # an input may repeat its rows
    assert torch.equal(q, q[:1, :1, :1].expand_as(q))


def test_one_token_with_any_stride():
    """One token whose stride along the tokens is 1, as a transposed column has it."""
    S, H, G = 2, 3, 2
    x = torch.randn(S, H, D, 1, device="cuda").half()
    c, d = (M.QuantCache(M.QuantParams(H, G, "fp16", "int8", 32), S, 64) for _ in range(2))
    c.append(x.transpose(2, 3), x.transpose(2, 3))
    d.append(x[..., 0], x[..., 0])
    assert torch.equal(c.k_tail[:, :, 0], d.k_tail[:, :, 0]) and torch.equal(c.v_tail[..., 0], d.v_tail[..., 0])
    y = torch.randn(S, D, 1, 1, device="cuda").half().permute(0, 2, 3, 1)
    pos, inv = torch.full((S, 1), 9, dtype=torch.int32, device="cuda"), torch.ones(64, device="cuda")
    a, b = M.qk_norm_rope(y, y, pos, inv), M.qk_norm_rope(y.reshape(S, 1, 1, D).clone(), y.reshape(S, 1, 1, D).clone(), pos, inv)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_shares_past_32_bits_are_refused():
    """(They were cut to their lower halves: another share.)"""
    c = M.QuantCache(M.QuantParams(1, 1, "fp16", "int8", 32), 1, 64)
    q = torch.zeros(1, 1, D, dtype=torch.float16, device="cuda")
    for share in ((1, (1 << 32) + 10), ((1 << 32) + 1, 10), (1 << 31, 1 << 31)):
        with pytest.raises(ValueError):
            c.decode_selected(q, 1.0, share)
    c.decode_selected(q, 1.0, ((1 << 31) - 1, (1 << 31) - 1))


def test_scales_of_other_number_types():
    """Numbers as numpy and torch hold them, as MosaicCache.decode takes them."""
    c = M.QuantCache(M.QuantParams(1, 1, "fp16", "int8", 32), 1, 64)
    x = torch.randn(1, 1, 33, D, device="cuda").half()
    c.append(x, x)
    q = torch.randn(1, 1, D, device="cuda").half()
    want = c.decode(q, 0.125), c.decode_selected(q, 0.125)
    pos, inv, w = torch.ones(1, 33, dtype=torch.int32, device="cuda"), torch.ones(64, device="cuda"), torch.ones(D, device="cuda").half()
    y = x.transpose(1, 2)
    rope = M.qk_norm_rope(y, y, pos, inv, w, w, eps=0.25)
    for n in (np.float32, np.float64, torch.tensor):
        assert torch.equal(c.decode(q, n(0.125)), want[0]) and torch.equal(c.decode_selected(q, n(0.125)), want[1])
        assert all(torch.equal(a, b) for a, b in zip(M.qk_norm_rope(y, y, pos, inv, w, w, eps=n(0.25)), rope))
