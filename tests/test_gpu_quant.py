"""The 8-bit KV cache against a plain reference (tests/_quant.py): codes,
scales, bounds and selections are equal, attention is within the error that its
arithmetic allows (_quant.bound)."""
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


def tokens(g, *shape, dt, strong=8.0):
    x = torch.randn(*shape, D, generator=g)
    x[..., 5] *= strong
    return x.to(dt)


def make(fmt, dtype, block, S, H, G, cap, fill=None):
    """A cache whose unwritten parts hold `fill` in every byte (0xff: NaN scales, codes and 16-bit values)."""
    c = M.QuantCache(M.QuantParams(H, G, dtype, fmt, block), S, cap)
    if fill is not None:
        for n in c.TENSORS:
            if n != "lens":
                getattr(c, n).view(torch.uint8).fill_(fill)
    return c


def close(got, want, zmax, where):
    want = np.asarray(want)
    norm = np.linalg.norm(want)
    rel = np.linalg.norm(got.double().cpu().numpy() - want) / norm if norm else np.linalg.norm(got.double().cpu().numpy())
    assert rel < R.bound(zmax), f"{where}: rel {rel:.2e} of {R.bound(zmax):.2e}"


def same_state(c, pairs, fill):
    """Every tensor of the cache against the reference; what no token reached still holds `fill`."""
    p = c.params
    B, N = p.block, c.k_scale.shape[2]
    t = {n: x.cpu() for n, x in c.tensors().items()}
    raw = lambda x: x.contiguous().view(torch.uint8).numpy()          # noqa: E731
    for (s, h), r in pairs.items():
        assert int(t["lens"][s, h]) == r.n, (s, h)
        for b in range(N):
            at = (s, h, b)
            if b < r.nb:
                for n, (code, scale) in (("k", r.kc[b]), ("v", r.vc[b])):
                    got = t[n][at].float().double().numpy()
                    assert np.array_equal(got if n == "k" else got.T, code), (n, at)
                    assert t[n + "_scale"][at].item() == float(scale), (n, at)
                hi, lo, unit = r.bounds[b]
                assert np.array_equal(t["bounds"][at].numpy(), np.stack([hi, lo])), at
                assert t["bound_scale"][at].item() == float(unit), at
            else:
                for n in ("k", "v", "k_scale", "v_scale", "bound_scale", "bounds"):
                    assert (raw(t[n][at].reshape(-1)) == fill).all(), (n, at)
        rest = r.n - r.nb * B
        kt, vt = t["k_tail"][s, h], t["v_tail"][s, h].T
        assert torch.equal(kt[:rest].float(), torch.from_numpy(r.k[r.nb * B:])), (s, h)
        assert torch.equal(vt[:rest].float(), torch.from_numpy(r.v[r.nb * B:])), (s, h)


@pytest.mark.parametrize("fmt,dtype,block", FORMS)
def test_append_in_any_pieces(fmt, dtype, block):
    """Prompts, chunks and single tokens, ragged, from views of other layouts,
    around the ends of blocks: the same contents however they came."""
    B, S, H, dt = block, 7, 2, DT[dtype]
    cap = 6 * B
    steps = [[0, 1, B - 1, B, B + 1, 3 * B + 5, 2 * B], [0, 1, 1, B, 2 * B - 1, 0, 1], [0, 0, B, 1, 1, B + 7, 3],
             [0, 3, 2 * B - 1, 2, 2, 0, 2 * B - 4]] + [[0, 1, 1, 1, 1, 1, 0]] * 3
    g = torch.Generator().manual_seed(3)
    total = [sum(x[s] for x in steps) for s in range(S)]
    assert max(total) <= cap
    k, v = tokens(g, S, H, max(total), dt=dt), tokens(g, S, H, max(total), dt=dt, strong=1.0)
    c = make(fmt, dtype, block, S, H, 4, cap, 0xff)
    at = [0] * S
    for i, counts in enumerate(steps):
        m = max(counts)
        kc, vc = torch.full((S, H, m, D), float("nan"), dtype=dt), torch.full((S, H, m, D), float("nan"), dtype=dt)
        for s, n in enumerate(counts):                         # (rows behind a sequence's tokens are NaN)
            kc[s, :, :n], vc[s, :, :n] = k[s, :, at[s]: at[s] + n], v[s, :, at[s]: at[s] + n]
            at[s] += n
        kc, vc = kc.cuda(), vc.cuda()
        if i % 2:                                              # token-major, and every other row of a larger array
            kc = kc.transpose(1, 2).contiguous().transpose(1, 2)
            vc = torch.stack((vc, vc), 3).view(S, H, 2 * m, D)[:, :, ::2]
        if m == 1 and i % 2 == 0:
            kc, vc = kc[:, :, 0], vc[:, :, 0]
        c.append(kc, vc, torch.tensor(counts, dtype=torch.int32, device="cuda"))
    pairs = {(s, h): R.Pair(k[s, h, : total[s]], v[s, h, : total[s]], fmt, block) for s in range(S) for h in range(H)}
    same_state(c, pairs, 0xff)
    assert not c.refused.any()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_of_extreme_values(fmt):
    """Blocks of zeros, of values far below 2^-100's scale, of the type's
    largest, of one outlier that leaves the rest below half a step, of ties."""
    B, dt = 32, torch.bfloat16
    g = torch.Generator().manual_seed(9)
    x = tokens(g, 1, 1, 6 * B, dt=torch.float32)
    x[0, 0, 0:B] = 0.0
    x[0, 0, B: 2 * B] *= 1e-38
    x[0, 0, 2 * B: 3 * B] = torch.sign(x[0, 0, 2 * B: 3 * B]) * torch.finfo(dt).max
    x[0, 0, 3 * B] = 1e6
    x[0, 0, 4 * B: 5 * B] = torch.arange(B * D).view(B, D) % 255 / 2.0 - 63.5   # halves and quarters of a step
    x[0, 0, 4 * B, 0] = 127.0
    x = x.to(dt)
    c = make(fmt, "bf16", B, 1, 1, 1, 6 * B, 0)
    c.append(x.cuda(), x.flip(2).contiguous().cuda())
    same_state(c, {(0, 0): R.Pair(x[0, 0], x.flip(2)[0, 0], fmt, B)}, 0)


def test_append_without_room():
    """A sequence without room takes none of a call's tokens and is counted;
    the others take theirs.  Whole-batch appends past any room are refused."""
    B, S, H, dt = 32, 3, 2, torch.float16
    g = torch.Generator().manual_seed(1)
    k, v = tokens(g, S, H, 2 * B, dt=dt), tokens(g, S, H, 2 * B, dt=dt)
    c = make("e4m3", "fp16", B, S, H, 1, 2 * B - 5, 0xff)
    assert c.max_tokens == 2 * B
    n = torch.tensor([2 * B, B, 0], dtype=torch.int32, device="cuda")
    c.append(k.cuda(), v.cuda(), n)
    c.append(k[:, :, :1].cuda(), v[:, :, :1].cuda())
    c.append(k.cuda(), v.cuda(), torch.tensor([0, 2 * B - 1, -3], dtype=torch.int32, device="cuda"))
    assert c.refused.tolist() == [1, 1, 0] and c.lens.tolist() == [[2 * B] * H, [B + 1] * H, [1] * H]
    pairs = {}
    for h in range(H):
        pairs[0, h] = R.Pair(k[0, h], v[0, h], "e4m3", B)
        pairs[1, h] = R.Pair(torch.cat((k[1, h, :B], k[1, h, :1])), torch.cat((v[1, h, :B], v[1, h, :1])), "e4m3", B)
        pairs[2, h] = R.Pair(k[2, h, :1], v[2, h, :1], "e4m3", B)
    same_state(c, pairs, 0xff)
    with pytest.raises(M.MosaicError):
        c.append(torch.zeros(S, H, 2 * B + 1, D, dtype=dt, device="cuda"), torch.zeros(S, H, 2 * B + 1, D, dtype=dt, device="cuda"))
    c.reset([1, 1])
    assert c.lens.tolist() == [[2 * B] * H, [0] * H, [1] * H]
    c.reset(torch.tensor([2, 7, -1], device="cuda"))
    assert c.lens.tolist() == [[2 * B] * H, [0] * H, [0] * H]
    for bad in ([3], [-1], torch.tensor([True, False, False], device="cuda"), torch.tensor([0])):
        with pytest.raises(ValueError):
            c.reset(bad)
    assert c.lens.tolist() == [[2 * B] * H, [0] * H, [0] * H]
    c.reset()
    assert not c.lens.any()


def test_long_append_without_room():
    """The same where a call's blocks are many and the lengths follow in a launch
    of their own; a sequence with nothing to take beside them."""
    B, S, H, dt, n = 32, 3, 2, torch.bfloat16, 40 * 32 + 3
    g = torch.Generator().manual_seed(6)
    k, v = tokens(g, S, H, n, dt=dt), tokens(g, S, H, n, dt=dt)
    c = make("int8", "bf16", B, S, H, 1, 64 * B, 0xff)
    counts = torch.tensor([n, 0, n - 7], dtype=torch.int32, device="cuda")
    c.append(k.cuda(), v.cuda(), counts)
    c.append(k.cuda(), v.cuda(), torch.tensor([n, n, 64 * B - n + 8], dtype=torch.int32, device="cuda"))
    assert c.refused.tolist() == [1, 0, 1] and c.lens.tolist() == [[n] * H, [n] * H, [n - 7] * H]
    same_state(c, {(s, h): R.Pair(k[s, h, : n - 7 * (s == 2)], v[s, h, : n - 7 * (s == 2)], "int8", B) for s in range(S) for h in range(H)}, 0xff)


def test_two_caches_on_two_streams():
    """Calls on different caches overlap; each has a workspace of its own."""
    B, H, G, n, dt = 32, 2, 4, 9000, torch.float16
    g = torch.Generator().manual_seed(12)
    k, v, q = tokens(g, 1, H, n, dt=dt).cuda(), tokens(g, 1, H, n, dt=dt).cuda(), tokens(g, 1, H * G, dt=dt).cuda()
    caches = [make("e4m3", "fp16", B, 1, H, G, n, 0xff) for _ in range(2)]
    for c in caches:
        c.append(k, v)
    want = caches[0].decode(q, SCALE), caches[0].decode_selected(q, SCALE, (1, 5))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in caches], [[], []]
    for _ in range(20):
        for i, c in enumerate(caches):
            with torch.cuda.stream(streams[i]):
                got[i].append((c.decode(q, SCALE), c.decode_selected(q, SCALE, (1, 5))))
    torch.cuda.synchronize()
    for outs in got:
        for a, b in outs:
            assert torch.equal(a, want[0]) and torch.equal(b, want[1])


def edges(block):
    return [0, 1, block - 1, block, block + 1, 4 * block, 5 * block + block // 2, 9 * block - 1, 17 * block + 3]


@pytest.mark.parametrize("G", [1, 4, 5, 8])
@pytest.mark.parametrize("fmt,dtype,block", FORMS)
def test_decode_and_selection_at_the_edges(fmt, dtype, block, G):
    """Lengths around blocks and around the waves' turns, empty ones among them,
    in a cache whose unwritten parts are NaN."""
    lens, H, dt = edges(block), 2, DT[dtype]
    S = len(lens)
    g = torch.Generator().manual_seed(G)
    k, v = tokens(g, S, H, max(lens), dt=dt), tokens(g, S, H, max(lens), dt=dt, strong=1.0)
    q = tokens(g, S, H * G, dt=dt, strong=1.0)
    c = make(fmt, dtype, block, S, H, G, max(lens), 0xff)
    c.append(k.cuda(), v.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    out = c.decode(q.cuda(), SCALE)
    blocks = torch.empty_like(c.k_scale, dtype=torch.int32)
    shares = [(1, 10), (1, 3), (1, 1)]
    sel = []
    for share in shares:
        sel.append((c.decode_selected(q.cuda(), SCALE, share, blocks=blocks), blocks.cpu().clone(), share))
    assert torch.equal(sel[-1][0], out)                        # a selection of everything
    for s, L in enumerate(lens):
        for h in range(H):
            r = R.Pair(k[s, h, :L], v[s, h, :L], fmt, block)
            qs, at = q[s, h * G: (h + 1) * G].float().numpy(), slice(h * G, (h + 1) * G)
            want, zmax = r.attend(qs, SCALE)
            close(out[s, at], want, zmax, f"L={L} h={h}")
            for o, b, share in sel:
                picked = r.select(qs, *share)
                assert b[s, h].tolist() == picked + [-1] * (b.shape[2] - len(picked)), f"L={L} h={h} {share}"
                want, zmax = r.attend(qs, SCALE, picked)
                close(o[s, at], want, zmax, f"L={L} h={h} {share}")


@pytest.mark.parametrize("fmt,dtype,block", [("e4m3", "bf16", 32), ("int8", "fp16", 64)])
def test_decode_scales_that_differ(fmt, dtype, block):
    """Blocks and queries of very different magnitudes: value scales growing and
    falling by powers of 2^20 along a sequence, a query of 2^-30, one of zeros,
    one whose logits reach hundreds."""
    B, G, dt = block, 4, DT[dtype]
    n = 24 * B + 9
    g = torch.Generator().manual_seed(5)
    k, v = tokens(g, 1, 1, n, dt=dt, strong=1.0), tokens(g, 1, 1, n, dt=torch.float32)
    steps = torch.tensor([0, -7, 3, 8, -12, 9, 10, -3]) if dtype == "fp16" else torch.tensor([0, -20, 20, 40, -40, 60, -100, 7])
    v = (v * torch.exp2(steps[(torch.arange(n) // B) % 8].float())[:, None]).to(dt)
    q = tokens(g, 1, G, dt=torch.float32, strong=1.0)
    q[0, 1] *= 2.0 ** -10 if dtype == "fp16" else 2.0 ** -30
    q[0, 2] = 0.0
    q[0, 3] *= 30.0
    q = q.to(dt)
    c = make(fmt, dtype, block, 1, 1, G, n, 0xff)
    c.append(k.cuda(), v.cuda())
    out = c.decode(q.cuda(), SCALE)
    r = R.Pair(k[0, 0], v[0, 0], fmt, block)
    for h in range(G):
        want, zmax = r.attend(q[0, h: h + 1].float().numpy(), SCALE)
        close(out[0, h: h + 1], want, zmax, f"head {h}")


@pytest.mark.parametrize("fmt,dtype,block", FORMS)
def test_values_that_are_not_finite_stay_in_their_head(fmt, dtype, block):
    """An infinity or a NaN in a whole block or in the unfinished one spoils its
    own (sequence, kv head); the others are as without it, bit for bit."""
    B, H, G, dt = block, 2, 3, DT[dtype]
    n = 20 * B + 7
    g = torch.Generator().manual_seed(15)
    k, v, q = tokens(g, 4, H, n, dt=dt), tokens(g, 4, H, n, dt=dt), tokens(g, 4, H * G, dt=dt, strong=1.0)
    bad_k, bad_v = k.clone(), v.clone()
    bad_k[0, 0, 3 * B + 1, 7] = float("inf")
    bad_v[0, 1, 5 * B + 9, 100] = float("nan")
    bad_k[1, 0, n - 2, 3] = float("nan")
    bad_v[1, 1, n - 1, 0] = -float("inf")
    outs = []
    for kk, vv in ((k, v), (bad_k, bad_v)):
        c = make(fmt, dtype, B, 4, H, G, n, 0xff)
        c.append(kk.cuda(), vv.cuda())
        outs.append((c.decode(q.cuda(), SCALE), c.decode_selected(q.cuda(), SCALE, (1, 4))))
    for clean, spoilt in zip(*outs):
        assert torch.equal(clean[2:], spoilt[2:]) and torch.isfinite(clean).all()
    for s in range(2):
        for h in range(H):
            assert not torch.isfinite(outs[1][0][s, h * G: (h + 1) * G]).all()


def test_selection_ties_and_many_blocks():
    """Equal blocks are taken from the lowest on; a pair of more blocks than a
    workgroup has threads, and of as many different scores; every form of the
    selection (by the cache's room: keys in registers, or read again)."""
    B, G = 32, 3
    g = torch.Generator().manual_seed(2)
    for nb, cap in ((2500, 2500), (4200, 4200), (40, 40 * 1024), (700, 20 * 1024), (300, 900)):
        n = nb * B + 7
        k = tokens(g, 2, 1, n, dt=torch.bfloat16)
        k[0, 0, : nb * B] = k[0, 0, :B].repeat(nb, 1)          # sequence 0: every block the same
        k[0, 0, 5 * B: 6 * B] *= 4.0                           # but two
        k[0, 0, 33 * B: 34 * B] *= 4.0
        q = tokens(g, 2, G, dt=torch.bfloat16)
        c = make("e4m3", "bf16", B, 2, 1, G, cap * B + 7, 0)
        c.append(k.cuda(), k.cuda())
        blocks = torch.empty_like(c.k_scale, dtype=torch.int32)
        out = c.decode_selected(q.cuda(), SCALE, (1, 16), blocks=blocks)
        for s in range(2):
            r = R.Pair(k[s, 0], k[s, 0], "e4m3", B)
            picked = r.select(q[s].float().numpy(), 1, 16)
            got = blocks[s, 0].cpu().tolist()
            assert got[: len(picked)] == picked and set(got[len(picked):]) == {-1}, (nb, s)
            want, zmax = r.attend(q[s].float().numpy(), SCALE, picked)
            close(out[s], want, zmax, f"{nb} blocks, sequence {s}")


@pytest.mark.parametrize("S,H,long", [(70, 1, 6000), (130, 3, 6000), (3, 8, 6000), (129, 1, 11000), (300, 1, 900)])
def test_uneven_batches_share_the_work(S, H, long):
    """Many short sequences, empty ones and long ones: the runs of every pair
    are found and joined."""
    B, G, dt = 32, 2, torch.float16
    lens = [0 if s % 9 == 4 else (long + s if s in (1, S - 1) else 5 * s % 97) for s in range(S)]
    g = torch.Generator(device="cuda").manual_seed(S)
    k, v = (torch.randn(S, H, max(lens), D, generator=g, device="cuda").to(dt) for _ in range(2))
    q = torch.randn(S, H * G, D, generator=g, device="cuda").to(dt)
    c = make("int8", "fp16", B, S, H, G, max(lens), 0xff)
    c.append(k, v, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    out, part = c.decode(q, SCALE), c.decode_selected(q, SCALE, (1, 5))
    for s in [s for s in range(S) if lens[s] > 800 or s % 13 == 0 or s % 9 == 4]:
        for h in range(H):
            r = R.Pair(k[s, h, : lens[s]].cpu(), v[s, h, : lens[s]].cpu(), "int8", B)
            qs, at = q[s, h * G: (h + 1) * G].float().cpu().numpy(), slice(h * G, (h + 1) * G)
            want, zmax = r.attend(qs, SCALE)
            close(out[s, at], want, zmax, f"s={s} h={h}")
            want, zmax = r.attend(qs, SCALE, r.select(qs, 1, 5))
            close(part[s, at], want, zmax, f"s={s} h={h} selected")


@pytest.mark.parametrize("H,nb,G", [(1, 5000, 8), (1, 1500, 1), (2, 700, 5), (1, 300, 3), (1, 250, 2)])
def test_pairs_of_many_runs(H, nb, G):
    """Few pairs take the whole chip: their runs are joined at once up to 32, in
    groups of 8, 16 and 32 beyond; the same every time."""
    B, n = 32, nb * 32 + 5
    g = torch.Generator().manual_seed(nb)
    k, v, q = tokens(g, 1, H, n, dt=torch.bfloat16), tokens(g, 1, H, n, dt=torch.bfloat16, strong=1.0), tokens(g, 1, H * G, dt=torch.bfloat16)
    c = make("e4m3", "bf16", B, 1, H, G, n, 0xff)
    c.append(k.cuda(), v.cuda())
    out = c.decode(q.cuda(), SCALE)
    for _ in range(3):
        assert torch.equal(c.decode(q.cuda(), SCALE), out)
    for h in range(H):
        want, zmax = R.Pair(k[0, h], v[0, h], "e4m3", B).attend(q[0, h * G: (h + 1) * G].float().numpy(), SCALE)
        close(out[0, h * G: (h + 1) * G], want, zmax, f"head {h}")


def test_codes_behind_four_gibibytes():
    """The second head's codes start behind byte 2^32 of the array."""
    B, G, cap = 64, 4, (1 << 25) + 64
    c = M.QuantCache(M.QuantParams(2, G, "bf16", "e4m3", B), 1, cap)
    g = torch.Generator().manual_seed(4)
    k, v, q = tokens(g, 1, 2, 5 * B + 3, dt=torch.bfloat16), tokens(g, 1, 2, 5 * B + 3, dt=torch.bfloat16), tokens(g, 1, 2 * G, dt=torch.bfloat16)
    c.append(k.cuda(), v.cuda())
    out, part = c.decode(q.cuda(), SCALE), c.decode_selected(q.cuda(), SCALE, (2, 5))
    for h in range(2):
        r, qs = R.Pair(k[0, h], v[0, h], "e4m3", B), q[0, h * G: (h + 1) * G].float().numpy()
        want, zmax = r.attend(qs, SCALE)
        close(out[0, h * G: (h + 1) * G], want, zmax, f"head {h}")
        want, zmax = r.attend(qs, SCALE, r.select(qs, 2, 5))
        close(part[0, h * G: (h + 1) * G], want, zmax, f"head {h} selected")


def test_results_repeat():
    B, S, H, G = 32, 3, 4, 7
    g = torch.Generator().manual_seed(8)
    k, v, q = (tokens(g, S, H, 9000, dt=torch.bfloat16).cuda() for _ in range(2)), None, tokens(g, S, H * G, dt=torch.bfloat16).cuda()
    k, v = k
    c = make("e4m3", "bf16", B, S, H, G, 9000)
    c.append(k, v)
    first = c.decode(q, SCALE), c.decode_selected(q, SCALE, (1, 7))
    for _ in range(5):
        assert torch.equal(c.decode(q, SCALE), first[0]) and torch.equal(c.decode_selected(q, SCALE, (1, 7)), first[1])


def _step(c, qkv, inv, w, H, G, select):
    S = qkv.shape[0]
    x = qkv.view(S, 1, (G + 2) * H, D)
    q, k, v = M.qk_norm_rope(x[:, :, : G * H], x[:, :, G * H: G * H + H], c.lens[:, :1], inv, w, w, v=x[:, :, G * H + H:])
    c.append(k, v)
    return c.decode_selected(q[:, 0], SCALE, select) if select else c.decode(q[:, 0], SCALE)


@pytest.mark.parametrize("select", [None, (1, 4)])
def test_steps_together_captured_and_eager(select):
    """A prompt, then steps of norm and rotation, append and attention: a
    captured step, replayed with new inputs and with the program's own work in
    between, follows the lengths on the device and gives what eager steps give;
    two graphs of two caches alternate."""
    S, H, G, B, steps = 3, 2, 4, 32, 40
    dt = torch.bfloat16
    g = torch.Generator().manual_seed(11)
    prompt = [0, 25, 300]
    inv = torch.pow(10000.0, -torch.arange(0, D, 2).float() / D).cuda()
    w = torch.ones(D, dtype=dt, device="cuda")
    k, v = tokens(g, S, H, 300, dt=dt).cuda(), tokens(g, S, H, 300, dt=dt).cuda()
    new = tokens(g, steps, S, (G + 2) * H, dt=dt, strong=1.0).flatten(2).cuda()
    n = torch.tensor(prompt, dtype=torch.int32, device="cuda")
    caches = [make("e4m3", "bf16", B, S, H, G, 300 + steps, 0xff) for _ in range(3)]
    for c in caches:
        c.append(k, v, n)
    want = [_step(caches[0], new[t], inv, w, H, G, select) for t in range(steps)]
    graphs = []
    for c in caches[1:]:
        x = new[0].clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):                          # a first step on another stream, then its capture
            first = _step(c, x, inv, w, H, G, select)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(first, want[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = _step(c, x, inv, w, H, G, select)
        graphs.append((graph, x, y))
    for t in range(1, steps):
        for graph, x, y in graphs:
            x.copy_(new[t])
            graph.replay()
        if t % 7 == 0:
            torch.cuda.synchronize()
            new.float().sum().item()
        for _, _, y in graphs:
            assert torch.equal(y, want[t]), f"step {t}"
    for c in caches:
        assert c.lens.tolist() == [[p + steps] * H for p in prompt]
    # the last step against the reference, from the tokens that the caches took
    c, t = caches[0], steps - 1
    x = new.view(steps, S, (G + 2) * H, D)
    for s in range(S):
        pos = (prompt[s] + torch.arange(steps, dtype=torch.int32, device="cuda"))[None]
        qr, kr, vr = M.qk_norm_rope(x[:, s, : G * H][None], x[:, s, G * H: G * H + H][None], pos, inv, w, w, v=x[:, s, G * H + H:][None])
        for h in range(H):
            kk, vv = torch.cat((k[s, h, : prompt[s]], kr[0, h])).cpu(), torch.cat((v[s, h, : prompt[s]], vr[0, h])).cpu()
            r, qs = R.Pair(kk, vv, "e4m3", B), qr[0, t, h * G: (h + 1) * G].float().cpu().numpy()
            o, zmax = r.attend(qs, SCALE, r.select(qs, *select) if select else None)
            close(want[t][s, h * G: (h + 1) * G], o, zmax, f"s={s} h={h}")


def test_refusals():
    c = make("e4m3", "bf16", 32, 2, 2, 4, 64)
    q = torch.zeros(2, 8, D, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(2, 2, 3, D, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(format="int4"), dict(block=16), dict(dtype="fp32"), dict(group_size=9), dict(num_kv_heads=0)):
        with pytest.raises((ValueError, M.MosaicError)):
            M.QuantCache(M.QuantParams(**bad), 1, 64)
    with pytest.raises(ValueError):
        M.QuantCache(M.QuantParams(), 0, 64)
    with pytest.raises(ValueError):
        M.QuantCache(M.QuantParams(), 1, 64, tensors={"keys": k})
    with pytest.raises(ValueError):
        M.QuantCache(M.QuantParams(2, 4, "bf16", "e4m3", 32), 2, 64, tensors={"lens": torch.zeros(2, dtype=torch.int32, device="cuda")})
    for call in (lambda: c.append(k.half(), k.half()), lambda: c.append(k, k[:, :, :2]), lambda: c.append(k[:1], k[:1]),
                 lambda: c.append(k.cpu(), k.cpu()), lambda: c.append(k, k, torch.ones(2, device="cuda")),
                 lambda: c.append(k, k, torch.ones(3, dtype=torch.int32, device="cuda")),
                 lambda: c.append(k.transpose(2, 3).contiguous().transpose(2, 3), k),
                 lambda: c.decode(q.half(), SCALE), lambda: c.decode(q[:, :4], SCALE), lambda: c.decode(q.cpu(), SCALE),
                 lambda: c.decode(q, SCALE, out=torch.empty(2, 8, D, dtype=torch.bfloat16, device="cuda")),
                 lambda: c.decode_selected(q, SCALE, blocks=torch.empty(2, 2, 1, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    odd = torch.zeros(2 * 2 * 3 * (D + 4), dtype=torch.bfloat16, device="cuda").view(2, 2, 3, D + 4)
    for call in (lambda: c.append(odd[..., :D], k), lambda: c.decode_selected(q, SCALE, (0, 10)), lambda: c.decode_selected(q, SCALE, (3, 2))):
        with pytest.raises(M.MosaicError):
            call()
    c.append(k[:, :, :0], k[:, :, :0])
    assert not c.lens.any() and not c.decode(q, SCALE).any() and not c.decode_selected(q, SCALE).any()
