"""One workspace for several caches: of other shapes and of other kinds, called in
turn, eager and captured; and the workspaces that are refused."""
import pytest
import torch

import paper_2607_00760_amd as M
from test_gpu_quant4 import DT, SCALE, fill, make, queries, tokens

pytestmark = pytest.mark.gpu

#            S  H  G  dtype  block  tokens  new
SHAPES = [(1, 1, 4, "bf16", 64, 6000, 5), (5, 3, 7, "fp16", 32, 900, 40), (300, 1, 1, "bf16", 32, 130, 3), (1, 2, 8, "bf16", 64, 200, 9)]


def one(shape, seed, **kw):
    """A cache with its queries, and (the same cache's) results on a workspace of its own."""
    S, H, G, dtype, block, n, new = shape
    k, v = tokens(S, H, n, DT[dtype], seed)
    c = make(S, H, G, dtype, block, n)
    fill(c, k, v, [n - 3 * (s % 5) for s in range(S)])
    q = queries(S, H * G, DT[dtype], seed + 1, new).cuda()
    want = c.decode(q[:, 0].contiguous(), SCALE), c.attend(q, SCALE)
    return c, q, want


def test_one_workspace():
    made = [one(s, 200 + 2 * i) for i, s in enumerate(SHAPES)]
    largest = max((c.workspace for c, _, _ in made), key=lambda w: w.numel())
    k, v = tokens(2, 2, 3000, torch.float16, 220)
    eight = M.QuantCache(M.QuantParams(2, 4, "fp16", "e4m3", 32), 2, 3000)
    fill(eight, k, v, [3000, 1700])
    q8 = queries(2, 8, torch.float16, 221).cuda()
    want8 = eight.decode(q8, SCALE), eight.decode_selected(q8, SCALE)
    space = torch.zeros(max(largest.numel(), eight.workspace.numel()) + 77, dtype=torch.uint8, device="cuda")
    shared = [M.Quant4Cache(c.params, c.num_seqs, c.max_tokens, tensors=c.tensors(), workspace=space) for c, _, _ in made]
    eight = M.QuantCache(eight.params, 2, 3000, tensors=eight.tensors(), workspace=space)
    assert all(c.workspace is space for c in shared + [eight])

    def step():
        out = []
        for c, (_, q, _) in zip(shared, made):
            out += [c.decode(q[:, 0].contiguous(), SCALE), c.attend(q, SCALE), eight.decode(q8, SCALE), eight.decode_selected(q8, SCALE)]
        return out
    want = [t for _, _, w in made for t in (*w, *want8)]
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(step(), want))
        assert not space[: 1 << 19].any()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(4):
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(c, b) for a, b, c in zip(out, want, eager))
        assert not space[: 1 << 19].any()


def test_workspaces_that_are_refused():
    p = M.Quant4Params(2, 4, "bf16", 64)
    c = M.Quant4Cache(p, 1, 1000)
    n = c.workspace.numel()
    space = torch.zeros(2 * n + 256, dtype=torch.uint8, device="cuda")
    for bad in (space[: n - 1], space[1:], space[128:], space[::2], space.cpu(), space.view(torch.int8), n):
        with pytest.raises((ValueError, TypeError)):
            M.Quant4Cache(p, 1, 1000, workspace=bad)
    M.Quant4Cache(p, 1, 1000, workspace=space[256: 256 + n])
    small = M.Quant4Cache(p, 1, 64)
    assert small.workspace.numel() < n
    with pytest.raises(ValueError):
        M.Quant4Cache(p, 1, 1000, workspace=small.workspace)
