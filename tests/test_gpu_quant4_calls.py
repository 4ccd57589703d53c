"""Calls around the 4-bit KV cache that a program makes: a run of its operators
together, eager and captured, values of any size, values that are not finite,
offsets past 32 bits, refusals."""
import math

import numpy as np
import pytest
import torch

import _quant4 as Q4
import paper_2607_00760_amd as M
from test_gpu_quant4 import DT, SCALE, fill, make, pairs, queries, tokens

pytestmark = pytest.mark.gpu
D = 128


def check_decode(out, ref, q, G, scale=SCALE):
    out = out.cpu().double().numpy()
    for s, row in enumerate(ref):
        for h, p in enumerate(row):
            want, tol = p.decode(q[s, h * G: (h + 1) * G].float().cpu().numpy(), scale)
            err = np.abs(out[s, h * G: (h + 1) * G] - want).max()
            assert err <= tol, (s, h, err, tol)


def check_attend(out, ref, q, G, m, scale=SCALE, causal=True):
    got = out.cpu().double().numpy()
    for s, row in enumerate(ref):
        for h, p in enumerate(row):
            last = np.repeat(p.n - m[s] + np.arange(m[s]) if causal else np.full(m[s], p.n - 1), G)
            x = q[s, : m[s], h * G: (h + 1) * G].reshape(-1, D).float().cpu().numpy()
            want, tol = p.attend(x, scale, last)
            err = np.abs(got[s, : m[s], h * G: (h + 1) * G].reshape(-1, D) - want)
            assert (err <= tol).all(), (s, h, err.max())


def step(c, qkv, at, inv, w, G, H, axes, n):
    """What a layer does with n new tokens of each sequence."""
    S = qkv.shape[0]
    x = qkv.view(S, n, (G + 2) * H, D)
    q, k, v = M.qk_norm_rope(x[:, :, : G * H], x[:, :, G * H: G * H + H], at, inv, w, w, v=x[:, :, G * H + H:], axes=axes)
    c.append(k, v)
    return c.decode(q[:, 0], SCALE) if n == 1 else c.attend(q, SCALE)


@pytest.mark.parametrize("n,dtype", [(1, "bf16"), (1, "fp16"), (3, "bf16"), (20, "fp16")])
def test_generation(n, dtype):
    """Norm and rotation on three axes, append and attention, step by step: a
    captured step, replayed with new inputs and with the program's own work in
    between, follows the lengths on the device and gives what eager steps give;
    graphs of two caches alternate."""
    S, H, G, B, steps, dt = 3, 2, 4, 32, 24, DT[dtype]
    prompt = [0, 25, 300]
    k, v = tokens(S, H, 300, dt, 31)
    g = torch.Generator().manual_seed(32)
    new = torch.randn((steps, S, n * (G + 2) * H * D), generator=g).to(dt).cuda()
    inv = torch.pow(10000.0, -torch.arange(0, D, 2).float() / D).cuda()
    w = torch.ones(D, dtype=dt, device="cuda")
    axes = bytes(i % 3 for i in range(64))
    at = torch.randint(0, 500, (steps, 3, S, n), generator=g).to(torch.int32).cuda()
    caches = [make(S, H, G, dtype, B, 300 + steps * n) for _ in range(3)]
    for c in caches:
        fill(c, k, v, prompt)
    want = [step(caches[0], new[t], at[t], inv, w, G, H, axes, n) for t in range(steps)]
    graphs = []
    for c in caches[1:]:
        x, pos = new[0].clone(), at[0].clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):                          # a first step on another stream, then its capture
            first = step(c, x, pos, inv, w, G, H, axes, n)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(first, want[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = step(c, x, pos, inv, w, G, H, axes, n)
        graphs.append((graph, x, pos, y))
    for t in range(1, steps):
        for graph, x, pos, _ in graphs:
            x.copy_(new[t])
            pos.copy_(at[t])
            graph.replay()
        if t % 7 == 0:
            torch.cuda.synchronize()
            new.float().sum().item()
        for *_, y in graphs:
            assert torch.equal(y, want[t]), f"step {t}"
    for c in caches:
        assert c.lens.tolist() == [[p + steps * n] * H for p in prompt]
        for name, t in c.tensors().items():
            if name in ("k", "v", "lens"):
                assert torch.equal(t, getattr(caches[0], name)), name
    # the last step against the reference, from the tokens that the caches took
    x = new.view(steps, S, n, (G + 2) * H, D)
    kk, vv, last = [[k[s, :, : prompt[s]]] for s in range(S)], [[v[s, :, : prompt[s]]] for s in range(S)], None
    for t in range(steps):
        last, kr, vr = M.qk_norm_rope(x[t][:, :, : G * H], x[t][:, :, G * H: G * H + H], at[t], inv, w, w, v=x[t][:, :, G * H + H:], axes=axes)
        for s in range(S):
            kk[s].append(kr[s].cpu())
            vv[s].append(vr[s].cpu())
    ref = [[Q4.Pair(torch.cat(kk[s], 1)[h], torch.cat(vv[s], 1)[h], B) for h in range(H)] for s in range(S)]
    if n == 1:
        check_decode(want[-1], ref, last[:, 0], G)
    else:
        check_attend(want[-1], ref, last, G, [n] * S)
    back = caches[0].read(300 + steps * n)
    for s in range(S):
        for h in range(H):
            for have, wanted in zip(back, ref[s][h].read()):
                assert torch.equal(have[s, h, : wanted.shape[0]].cpu(), wanted)


def test_a_chunk_is_its_tokens():
    """Queries of a chunk attend what they attend alone, and with others behind them."""
    S, H, G, B, n = 1, 2, 4, 64, 70
    k, v = tokens(S, H, 500, torch.float16, 33)
    c = make(S, H, G, "fp16", B, 640)
    fill(c, k, v, [500])
    q = queries(S, H * G, torch.float16, 34, n).cuda()
    out = c.attend(q, SCALE)
    assert torch.equal(c.attend(q, SCALE, out=q.clone()), out)
    mine = q.clone()
    assert c.attend(mine, SCALE, out=mine) is mine and torch.equal(mine, out)          # in place
    check_attend(out, pairs(k, v, [500], B), q, G, [n])
    tail = c.attend(q[:, -3:], SCALE)
    check_attend(tail, pairs(k, v, [500], B), q[:, -3:], G, [3])


@pytest.mark.parametrize("scale", [0.0, -SCALE, 3e-5, 4.0])
@pytest.mark.parametrize("dtype,block,G", [("fp16", 32, 7), ("bf16", 64, 4)])
def test_softmax_scales(dtype, block, G, scale):
    lens = [0, 5, 64, 333]
    k, v = tokens(4, 2, 333, DT[dtype], 35)
    c = make(4, 2, G, dtype, block, 400)
    fill(c, k, v, lens)
    ref = pairs(k, v, lens, block)
    q = queries(4, 2 * G, DT[dtype], 36)
    check_decode(c.decode(q.cuda(), scale), ref, q, G, scale)
    for n in (2, 50):
        q = queries(4, 2 * G, DT[dtype], 37, n)
        check_attend(c.attend(q.cuda(), scale), ref, q, G, [n] * 4, scale)


@pytest.mark.parametrize("power", [-90, -60, 0, 60, 100, 126])
def test_bf16_values_of_any_size(power):
    """V from 2^-90 to the type's largest, in blocks and in the tail, with sizes
    apart between tokens; its sums stay in range, and what is small is exact."""
    S, H, G, B, n = 1, 2, 4, 64, 1000
    k, v = tokens(S, H, n, torch.bfloat16, 38)
    v = (v.float().clamp(-1.9, 1.9) * 2.0 ** power).bfloat16()
    v[:, :, ::5] = (v[:, :, ::5].float() * 2.0 ** -30).bfloat16()
    for L in (n, 960, 40):
        c = make(S, H, G, "bf16", B, n)
        fill(c, k, v, [L])
        q = queries(S, H * G, torch.bfloat16, 39)
        check_decode(c.decode(q.cuda(), SCALE), pairs(k[:, :, :L], v[:, :, :L], [L], B), q, G)


def test_weight_on_tokens_of_small_values():
    """Almost all weight on tokens whose values are 2^-40 of the others': the
    others' share of the output is as exact as they are large."""
    n, B = 256, 64
    k = torch.zeros((1, 1, n, D))
    k[..., 0] = torch.where(torch.arange(n) % 2 == 0, 20.0, -20.0)
    v = torch.randn((1, 1, n, D), generator=torch.Generator().manual_seed(40))
    v[:, :, ::2] *= 2.0 ** -40
    q = torch.zeros((1, 1, D))
    q[..., 0] = 6.0
    for dt in (torch.bfloat16, torch.float16):
        kd, vd, qd = k.to(dt), v.to(dt), q.to(dt)
        c = make(1, 1, 1, "bf16" if dt == torch.bfloat16 else "fp16", B, n)
        fill(c, kd, vd, [n])
        for scale in (0.02, 0.1, 0.15):
            pair = Q4.Pair(kd[0, 0], vd[0, 0], B)
            want, _ = pair.decode(qd[0].float().numpy(), scale)
            got = c.decode(qd.cuda(), scale).cpu().double().numpy()[0]
            # A weight is off by its logit's roundings, values' sums by theirs: 2^-18 of
            # the largest channel.  As fp16 numbers the small values are zeros, on a grid
            # of the least scale s = 2^-19: such a token adds p (zero + 8 s) and takes
            # p s (0 - 8), which has the 22 bits of its weight's two parts; the
            # difference is up to 2^-22 of 8 p s, summed over the tokens, and the sums'
            # roundings are as much.
            z = qd[0].double().numpy() @ pair.held()[0].T * scale
            w = np.exp(z - z.max())
            w = w / w.sum() * np.concatenate([s for _, s, _ in pair.vc])
            assert np.abs(got - want).max() <= 2.0 ** -18 * np.abs(want).max() + 2.0 ** -21 * 8 * w.sum(), (dt, scale)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["k block", "v block", "k tail", "v tail"])
def test_values_that_are_not_finite_stay_in_their_head(bad, where):
    S, H, G, B, n = 2, 2, 4, 32, 70
    k, v = tokens(S, H, n, torch.bfloat16, 41)
    x = k if where[0] == "k" else v
    x[1, 0, 40 if "block" in where else 66, 9] = bad
    c = make(S, H, G, "bf16", B, n)
    fill(c, k, v, [n, n])
    q = queries(S, H * G, torch.bfloat16, 42, 4)
    one, some = c.decode(q[:, 3].contiguous().cuda(), SCALE), c.attend(q.cuda(), SCALE)
    rows = torch.zeros(S, H * G, dtype=torch.bool)
    rows[1, :G] = True
    # what a key's NaN or a value's reaches shows; an infinite key may take all weight or none
    if not (where == "k tail" and math.isinf(bad)):
        assert not one.cpu()[rows].isfinite().all(-1).any()
        assert not some.cpu()[:, 3][rows].isfinite().all(-1).any()
    ref = pairs(torch.nan_to_num(k, 0, 0, 0), torch.nan_to_num(v, 0, 0, 0), [n, n], B)
    for s in range(S):
        for h in range(H):
            if (s, h) == (1, 0):
                continue
            want, tol = ref[s][h].decode(q[s, 3, h * G: (h + 1) * G].float().numpy(), SCALE)
            assert np.abs(one[s, h * G: (h + 1) * G].cpu().double().numpy() - want).max() <= tol
            assert some[s, :, h * G: (h + 1) * G].isfinite().all()
    kb, vb = c.read(n)
    assert torch.equal(kb[0].cpu(), torch.stack([ref[0][h].read()[0] for h in range(H)]))
    assert torch.equal(vb[0].cpu(), torch.stack([ref[0][h].read()[1] for h in range(H)]))


def test_appends_without_room():
    S, H, B = 3, 2, 32
    k, v = tokens(S, H, 100, torch.float16, 43)
    c = make(S, H, 4, "fp16", B, 64)
    fill(c, k, v, [60, 10, 64])
    before = {n: t.clone() for n, t in c.tensors().items()}
    c.append(k[:, :, :5].cuda(), v[:, :, :5].cuda())
    assert c.refused.tolist() == [1, 0, 1] and c.lens.tolist() == [[60] * H, [15] * H, [64] * H]
    for n, t in c.tensors().items():
        if n != "lens":
            assert torch.equal(t[0].view(torch.uint8), before[n][0].view(torch.uint8)) and \
                torch.equal(t[2].view(torch.uint8), before[n][2].view(torch.uint8)), n
    c.reset([1, 2])
    c.append(k[:, :, :4].cuda(), v[:, :, :4].cuda(), torch.tensor([9, -3, 2], dtype=torch.int32, device="cuda"))
    assert c.lens.tolist() == [[64] * H, [0] * H, [2] * H] and c.refused.tolist() == [1, 0, 1]
    with pytest.raises(M.MosaicError, match="CAPACITY"):
        c.append(k[:, :, :65].cuda(), v[:, :, :65].cuda())


def test_one_block_of_32():
    """A cache that holds less than a step of 64 tokens."""
    for n in (1, 31, 32):
        k, v = tokens(1, 1, n, torch.bfloat16, 44)
        c = make(1, 1, 4, "bf16", 32, 32)
        fill(c, k, v, [n])
        ref = pairs(k, v, [n], 32)
        for m in (1, 8, 60):
            q = queries(1, 4, torch.bfloat16, 45, m)
            check_attend(c.attend(q.cuda(), SCALE, causal=False), ref, q, 4, [m], causal=False)
        q = queries(1, 4, torch.bfloat16, 46)
        check_decode(c.decode(q.cuda(), SCALE), ref, q, 4)


def test_two_streams():
    """Two caches on two streams, many times over."""
    H, G, B, n = 2, 4, 64, 3000
    caches, qs, want, streams = [], [], [], []
    for i in range(2):
        k, v = tokens(1, H, n, torch.bfloat16, 50 + i)
        c = make(1, H, G, "bf16", B, n)
        fill(c, k, v, [n])
        q = queries(1, H * G, torch.bfloat16, 52 + i, 6).cuda()
        caches.append(c)
        qs.append(q)
        want.append((c.decode(q[:, 0].contiguous(), SCALE), c.attend(q, SCALE)))
        streams.append(torch.cuda.Stream())
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append((caches[i].decode(qs[i][:, 0].contiguous(), SCALE), caches[i].attend(qs[i], SCALE)))
    torch.cuda.synchronize()
    for i in range(2):
        for a, b in got[i]:
            assert torch.equal(a, want[i][0]) and torch.equal(b, want[i][1])


def test_offsets_past_32_bits():
    """Codes of 5 GB: the last heads lie past 2^32 bytes."""
    H, G, B, n = 64, 1, 64, 1 << 20
    n += 21
    c = M.Quant4Cache(M.Quant4Params(num_kv_heads=H, group_size=G, dtype="bf16", block=B), 1, n + 60)
    assert c.k.numel() > 1 << 32
    g = torch.Generator(device="cuda").manual_seed(53)
    for h in (0, H - 1):
        c.k[0, h].random_(0, 256, generator=g)
        c.v[0, h].random_(0, 256, generator=g)
    for t, lo in ((c.k_grid, -0.5), (c.v_grid, -1.0)):
        t[..., 0, :] = -lo / 8
        t[..., 1, :] = lo
    c.k_tail.normal_(generator=g)
    c.v_tail.normal_(generator=g)
    c.lens.fill_(n)
    for h in range(1, H - 1):
        c.k[0, h].zero_()
        c.v[0, h].zero_()
    x = torch.randn((1, H, 40, D), generator=g, device="cuda").bfloat16()
    c.append(x, -x)                                            # a block more is whole, 61 tokens of the tail become it
    n += 40
    assert (c.lens == n).all()
    start = n - 300
    k, v = c.read(300, start)
    nb = n // B
    for h in (0, H - 1):
        kk = c.k_grid[0, h, :, 1, None].float() + c.k_grid[0, h, :, 0, None].float() * Q4.unpack(c.k[0, h]).float()
        vv = c.v_grid[0, h, :, 1, :, None].float() + c.v_grid[0, h, :, 0, :, None].float() * Q4.unpack(c.v[0, h]).transpose(1, 2).float()
        kk = torch.cat((kk[:nb].flatten(0, 1), c.k_tail[0, h, : n % B].float()))
        vv = torch.cat((vv[:nb].flatten(0, 1), c.v_tail[0, h].T[: n % B].float()))
        assert torch.equal(k[0, h], kk[start:].bfloat16()) and torch.equal(v[0, h], vv[start:].bfloat16())
        assert torch.equal(k[0, h, -40:, 5][-(n % B):], x[0, h, -(n % B):, 5])
        q = torch.randn((1, 3, H * G, D), generator=g, device="cuda").bfloat16()
        one, some = c.decode(q[:, 2].contiguous(), SCALE), c.attend(q, SCALE)
        p = torch.softmax((q[0, 2, h].double() @ kk.double().T) * SCALE, 0)
        # a million weights of about 2^-20: their errors are 2^-24 of a logit's terms, at random
        assert (one[0, h] - p @ vv.double()).abs().max() <= 2.0 ** -18
        assert (some[0, 2, h] - p @ vv.double()).abs().max() <= 2.0 ** -8 * (p @ vv.double()).abs().max() + 2.0 ** -16


def test_refusals():
    c = make(2, 2, 4, "bf16", 32, 64, dirty=False)
    q = torch.zeros(2, 8, D, dtype=torch.bfloat16, device="cuda")
    qs = torch.zeros(2, 3, 8, D, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(2, 2, 3, D, dtype=torch.bfloat16, device="cuda")
    n = torch.ones(2, dtype=torch.int32, device="cuda")
    for bad in (dict(block=16), dict(dtype="fp32"), dict(group_size=9), dict(num_kv_heads=0)):
        with pytest.raises((ValueError, M.MosaicError)):
            M.Quant4Cache(M.Quant4Params(**bad), 1, 64)
    for args, kw in (((0, 64), {}), ((1, 0), {}), ((1, 64), dict(tensors={"keys": k})), ((1, 64), dict(tensors={"lens": n})), ((1, 64), dict(device="cpu"))):
        with pytest.raises(ValueError):
            M.Quant4Cache(M.Quant4Params(2, 4, "bf16", 32), *args, **kw)
    for call in (lambda: c.append(k.half(), k.half()), lambda: c.append(k, k[:, :, :2]), lambda: c.append(k, k, n.long()),
                 lambda: c.decode(q.half(), SCALE), lambda: c.decode(q[:, :4], SCALE), lambda: c.decode(q.cpu(), SCALE),
                 lambda: c.attend(q, SCALE), lambda: c.attend(qs.half(), SCALE), lambda: c.attend(qs[:, :, :4], SCALE), lambda: c.attend(qs.cpu(), SCALE),
                 lambda: c.attend(qs, SCALE, n[:1]), lambda: c.attend(qs, SCALE, n.long()), lambda: c.attend(qs, SCALE, out=qs[:, :2]),
                 lambda: c.attend(qs.transpose(2, 3).contiguous().transpose(2, 3), SCALE), lambda: c.read(-1), lambda: c.read(1 << 31),
                 lambda: c.read(3, n.long()), lambda: c.read(3, n[:1]), lambda: c.read(3, 1 << 31), lambda: c.read(3, 0, k[:, :, :2]),
                 lambda: c.read(3, 0, k, k.half())):
        with pytest.raises(ValueError):
            call()
    odd = torch.zeros(2 * 2 * 3 * (D + 4), dtype=torch.bfloat16, device="cuda").view(2, 2, 3, D + 4)[..., :D]
    same = torch.zeros(1, 1, 1, D, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: c.append(odd, k), lambda: c.read(3, 0, odd), lambda: c.read(3, 0, same.expand(2, 2, 3, D)),
                 lambda: c.attend(qs, SCALE, out=same.expand(2, 3, 8, D))):
        with pytest.raises(M.MosaicError):
            call()
    c.append(k[:, :, :0], k[:, :, :0])
    assert c.attend(qs[:, :0], SCALE).shape == (2, 0, 8, D) and c.read(0)[0].shape == (2, 2, 0, D)
    assert not c.lens.any() and not c.decode(q, SCALE).any() and not c.attend(qs, SCALE).any()
    assert not c.attend(qs, SCALE, torch.tensor([9, -1], dtype=torch.int32, device="cuda"), causal=False).any()
