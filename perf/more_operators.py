"""Timed cases of the operators around the 4-bit KV cache, with their plain forms.

  axes    queries and keys normalised per head and rotated to positions of
          several axes (time, height, width) in one pass (qk_norm_rope)
  fill    keys and values written into a cache of 4-bit codes, part by part,
          and read back (Quant4Cache.append, .read)
  read    a run of each sequence's tokens read back out of the 4-bit or the
          8-bit cache (Quant4Cache.read, QuantCache.read)
  decode  attention of one query token a sequence over the 4-bit cache
          (Quant4Cache.decode)
  attend  attention of several query tokens of a sequence over the 4-bit
          cache, causal or not (Quant4Cache.attend)

Plain forms compute in 32 bits from the same definitions, with elementary
torch operations; `exact` does so in 64 bits, apart from them.

Definitions.  T is the cache's 16-bit type, LEAST 2^-19 (fp16) or 2^-100
(bf16).  The grid of a row x of values: lo and hi its least and largest, scale
= the largest value of T that is not above (hi / 2 - lo / 2) / 7.5, or LEAST
where that is more, zero = lo; a value's code = nearest((x / 2 - lo / 2) * (2 /
scale)), 0 to 15, each step in 32 bits; it stands for zero + scale * code.  Whole blocks of B
tokens of one (sequence, kv head) are encoded: a row is a channel's keys over
the block's tokens, or a token's values over the channels.  Tokens past the
last whole block stay in 16 bits, in the tail.  What is read back is rounded
to T.  A query token of `decode` attends what the codes stand for; those of
`attend` what is read back, query i of a sequence's m being its token L - m + i.

The 4-bit cache is a set of tensors (S sequences, H kv heads, room for N blocks):
  k [S][H][N][B][64], v [S][H][N][128][B / 2]   uint8, two codes each (the first
                                                in the lower half): of channels, of tokens
  k_grid [S][H][N][2][128], v_grid [S][H][N][2][B]   T: scales, then zeros
  k_tail [S][H][B][128], v_tail [S][H][128][B]  T
  lens [S][H]                                   int32, tokens held
The 8-bit cache holds codes k [S][H][N][B][128] and v [S][H][N][128][B]
(float8_e4m3fn or int8) that stand for code * k_scale, v_scale [S][H][N], and
the same tails and lens.
"""
import math

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
EPS = 1e-6


def _case(name, op, seqs, n, **more):
    """n: tokens of a sequence (axes, fill), or in the cache (the others)."""
    c = dict(name=name, op=op, seqs=seqs, n=n, hkv=8, group=4, dtype="bf16", block=64, ragged=False)
    if op == "axes":
        c.update(rot=128, interleaved=False, norm=True, num_axes=3, spread=False)
    if op == "fill":
        c.update(parts=1)
    if op == "read":
        c.update(fmt="int4", take=n)
    if op == "attend":
        c.update(new=1, causal=True)
    c.update(more)
    return c


def listed():
    return [
        # one token of a batch, as every generated token takes it: latency
        _case("axes_b16_n1_bf16", "axes", 16, 1),
        # a batch of images and text, axes dealt to the pairs in turn
        _case("axes_b2_16k_fp16", "axes", 2, 16384, dtype="fp16", spread=True),
        # the prompts of an ordinary batch into the cache, and out of it again
        _case("fill_b4_32k_bf16", "fill", 4, 32785),
        # prompts of many lengths that arrive in three chunks
        _case("fill_b16_3x700_fp16", "fill", 16, 2100, hkv=4, group=7, dtype="fp16", block=32, ragged=True, parts=3),
        # contexts handed on in 16 bits, whole, and the last tokens of a ragged batch out of an 8-bit cache
        _case("read_b8_32k_fp16_int4", "read", 8, 32768, dtype="fp16"),
        _case("read_b16_ragged_bf16_e4m3", "read", 16, 32768, hkv=4, group=7, fmt="e4m3", block=32, ragged=True, take=5001),
        # one short sequence: the smallest attention step
        _case("decode_b1_4k_fp16", "decode", 1, 4117, dtype="fp16"),
        # the long-context batch
        _case("decode_b8_128k_bf16", "decode", 8, 131072),
        # a ragged serving batch of a 28-head model
        _case("decode_b16_ragged_g7_bf16", "decode", 16, 98304, hkv=4, group=7, block=32, ragged=True),
        # drafted tokens of a batch, checked at once
        _case("attend_b8_32k_5new_bf16", "attend", 8, 32773, new=5),
        # a chunk of a long prompt
        _case("attend_b1_32k_2048new_bf16", "attend", 1, 32768, new=2048),
        # queries of other lengths than the encoder's states that they attend
        _case("attend_b6_1500_448new_fp16", "attend", 6, 1500, hkv=12, group=1, dtype="fp16", block=32, ragged=True, new=448, causal=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["axes", "fill", "read", "decode", "decode", "attend", "attend"])
    hkv, group = rng.choice([(8, 4), (8, 4), (4, 7), (2, 8), (12, 1), (4, 5), (1, 3)])
    c = dict(op=op, hkv=hkv, group=group, dtype=rng.choice(["fp16", "bf16"]), block=rng.choice([32, 64]), ragged=False)
    seqs = rng.choice([1, 1, 2, 3, 4, 8, 16])
    most = {"axes": 2 * 16384 * 40, "fill": 4 * 32785 * 8, "read": 8 * 32768 * 8, "decode": 8 * 131072 * 8, "attend": 8 * 32773 * 8}[op]
    per = hkv * (group + 1) if op == "axes" else hkv
    top = min(most // (seqs * per), {"axes": 32768, "fill": 131072, "read": 262144, "decode": 1 << 19, "attend": 131072}[op])
    c.update(seqs=seqs, n=_log_int(rng, 1, top), ragged=seqs > 1 and rng.random() < 0.5)
    if op == "axes":
        c.update(ragged=False, rot=rng.choice([128, 128, 64, 96, 32]), interleaved=rng.random() < 0.4, norm=rng.random() < 0.7,
                 num_axes=rng.choice([2, 3, 3, 4]), spread=rng.random() < 0.5)
    elif op == "fill":
        c.update(parts=rng.choice([1, 1, 2, 3]))
    elif op == "read":
        c.update(fmt=rng.choice(["int4", "int4", "e4m3", "int8"]), take=_log_int(rng, 1, c["n"]))
    elif op == "attend":
        c.update(causal=rng.random() < 0.7)
        room = 2048 * 32768 * 32 // (c["n"] * seqs * hkv * group)
        # drafted tokens; a chunk or an encoder's queries
        c.update(new=rng.randint(1, 8) if rng.random() < 0.5 else _log_int(rng, 1, 2048))
        c["new"] = max(1, min(c["new"], room, c["n"] if c["causal"] else 2048))
    return c


# ---------------------------------------------------------------- inputs

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _spread(most, seqs, ragged):
    """Lengths: all `most`, or from most / 6 up to it."""
    if not ragged:
        return [most] * seqs
    lo = max(1, most // 6)
    return [most - (most - lo) * ((7 * i) % seqs) // seqs for i in range(seqs)]


def _lens(case):
    return _spread(case["n"], case["seqs"], case["ragged"])


def _new_lens(case):
    """Queries of each sequence; with causal ones at most its tokens."""
    m = _spread(case["new"], case["seqs"], case["ragged"])
    return [min(a, L) for a, L in zip(m, _lens(case))] if case["causal"] else m


def _axes(case):
    """Which axis turns each pair: in runs, or in turn."""
    half, A = case["rot"] // 2, case["num_axes"]
    return tuple(i % A if case["spread"] else i * A // half for i in range(half))


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, S, H, G, n = _dtype(case), case["seqs"], case["hkv"], case["group"], case["n"]
    d = {}

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    if case["op"] == "axes":
        d["q_weight"], d["k_weight"] = (1 + 0.2 * normal(D)).to(dt), (1 + 0.2 * normal(D)).to(dt)
        # the output of a fused projection: queries, keys and values of a token side by side
        qkv = torch.empty((S, n, (H * G + 2 * H) * D), dtype=dt, device="cuda")
        for s in range(S):
            qkv[s] = (2.0 * normal(n, qkv.shape[2])).to(dt)
        d["qkv"] = qkv
        # frames of 24 x 24 patches, one after the other
        t = torch.arange(n, device="cuda")[None] + torch.randint(0, 1 << 14, (S, 1), generator=gen, device="cuda")
        axes = [t // 576, t // 24 % 24, t % 24, t]
        d["positions"] = torch.stack(axes[: case["num_axes"]]).to(torch.int32)
        rot = case["rot"]
        d["inv_freq"] = torch.pow(torch.tensor(500000.0, dtype=torch.float64), -torch.arange(0, rot, 2, dtype=torch.float64) / rot).float().cuda()
        return d
    lens = _lens(case)
    d["lens"] = lens
    # normals; a few channels of a head's keys are strong and far from zero, a few of its values strong
    k, v = (torch.empty((S, H, n, D), dtype=dt, device="cuda") for _ in range(2))
    ks, kb, vs = torch.ones((H, D), device="cuda"), torch.zeros((H, D), device="cuda"), torch.ones((H, D), device="cuda")
    for h in range(H):
        at = torch.randperm(D, generator=gen, device="cuda")[:8]
        ks[h, at[:4]], kb[h, at[:4]], vs[h, at[4:]] = 4.0, 8.0, 3.0
    for s in range(S):
        k[s] = (normal(H, n, D) * ks[:, None] + kb[:, None]).to(dt)
        v[s] = (normal(H, n, D) * vs[:, None]).to(dt)
    d["k"], d["v"] = k, v
    if case["op"] == "fill":
        # how many tokens of each sequence a part brings; the parts follow one another
        d["cuts"] = [[L * i // case["parts"] for L in lens] for i in range(case["parts"] + 1)]
    if case["op"] == "decode":
        q = normal(S, H * G, D)
        d["q"] = q.to(dt)
        # some tokens in twenty lie along their group's queries
        u = q.view(S, H, G, D).sum(2)
        u = 6.0 * u / u.norm(dim=-1, keepdim=True)
        for s in range(S):
            hot = torch.rand(n, generator=gen, device="cuda") < 0.05
            k[s, :, hot] = (k[s, :, hot].float() + u[s][:, None, :]).to(dt)
    if case["op"] == "attend":
        d["q"] = normal(S, case["new"], H * G, D).to(dt)
        d["new_lens"] = _new_lens(case)
    if case["op"] == "read":                                   # the last tokens of each sequence
        d["starts"] = [L - min(L, case["take"]) for L in lens]
    return d


def _fmt(case):
    return case.get("fmt", "int4")


def _empty_cache(case, cap):
    S, H, B, dt = case["seqs"], case["hkv"], case["block"], _dtype(case)
    N = -(-cap // B)

    def zeros(*shape, dtype=torch.float32):
        return torch.zeros((S, H) + shape, dtype=dtype, device="cuda")
    c = dict(k_tail=zeros(B, D, dtype=dt), v_tail=zeros(D, B, dtype=dt), lens=zeros(dtype=torch.int32))
    if _fmt(case) == "int4":
        return dict(k=zeros(N, B, D // 2, dtype=torch.uint8), v=zeros(N, D, B // 2, dtype=torch.uint8), k_grid=zeros(N, 2, D, dtype=dt),
                    v_grid=zeros(N, 2, B, dtype=dt), **c)
    code = torch.float8_e4m3fn if _fmt(case) == "e4m3" else torch.int8
    return dict(k=zeros(N, B, D, dtype=torch.int8).view(code), v=zeros(N, D, B, dtype=torch.int8).view(code), k_scale=zeros(N),
                v_scale=zeros(N), bound_scale=zeros(N), bounds=zeros(N, 2, D, dtype=torch.int8), **c)


def prepare(case, seed):
    d = _inputs(case, seed)
    d["case"] = case
    S, H, G, dt = case["seqs"], case["hkv"], case["group"], _dtype(case)
    if case["op"] == "axes":
        x = d["qkv"].view(S, case["n"], H * G + 2 * H, D)
        d["split"] = x[:, :, : H * G], x[:, :, H * G: H * G + H], x[:, :, H * G + H:]
        d["axes"] = _axes(case)
        return d
    d["lens_dev"] = torch.tensor(d["lens"], dtype=torch.int32, device="cuda")
    d["cache"] = _empty_cache(case, case["n"])
    if case["op"] == "fill":
        d["chunks"] = []
        for a, b in zip(d["cuts"], d["cuts"][1:]):
            m = max(1, max(y - x for x, y in zip(a, b)))
            kc, vc = (torch.zeros((S, H, m, D), dtype=dt, device="cuda") for _ in range(2))
            for s in range(S):
                kc[s, :, : b[s] - a[s]], vc[s, :, : b[s] - a[s]] = d["k"][s, :, a[s]: b[s]], d["v"][s, :, a[s]: b[s]]
            d["chunks"].append((kc, vc, torch.tensor([y - x for x, y in zip(a, b)], dtype=torch.int32, device="cuda")))
        del d["k"], d["v"]
        d["out"] = [torch.zeros((S, H, case["n"], D), dtype=dt, device="cuda") for _ in range(2)]
    else:
        k, v = d.pop("k"), d.pop("v")
        for s in range(S):                                     # the cache holds the context from here on
            one = {x: t[s: s + 1] for x, t in d["cache"].items()}
            (_plain_append if _fmt(case) == "int4" else _fill8)(one, k[s: s + 1], v[s: s + 1], d["lens_dev"][s: s + 1])
    if case["op"] == "read":
        d["out"] = [torch.zeros((S, H, case["take"], D), dtype=dt, device="cuda") for _ in range(2)]
        d["starts_dev"] = torch.tensor(d["starts"], dtype=torch.int32, device="cuda")
    if case["op"] == "attend":
        d["new_dev"] = torch.tensor(d["new_lens"], dtype=torch.int32, device="cuda")
        d["out"] = torch.zeros_like(d["q"])
    if own:                                                    # the framework's handle on these tensors
        import paper_2607_00760_amd as mosaic
        shape = dict(num_kv_heads=H, group_size=G, dtype=case["dtype"], block=case["block"])
        if _fmt(case) == "int4":
            d["handle"] = mosaic.Quant4Cache(mosaic.Quant4Params(**shape), S, case["n"], tensors=d["cache"])
        else:
            d["handle"] = mosaic.QuantCache(mosaic.QuantParams(format=case["fmt"], **shape), S, case["n"], tensors=d["cache"])
    return d


def run(state):
    case = state["case"]
    op = case["op"]
    if op == "axes":
        return _run_axes(state)
    if op == "fill":
        return _run_fill(state)
    if op == "read":
        if own:
            return state["handle"].read(case["take"], state["starts_dev"], *state["out"])
        return _plain_read(state["cache"], case["take"], state["starts_dev"], *state["out"])
    if op == "decode":
        if own:
            return state["handle"].decode(state["q"], SCALE)
        return _plain_decode(state["cache"], state["q"], case["group"])
    if own:
        return state["handle"].attend(state["q"], SCALE, state["new_dev"], causal=case["causal"], out=state["out"])
    return _plain_attend(state["cache"], state["q"], case["group"], state["new_dev"], case["causal"], state["out"])


def _run_axes(state):
    case, (q, k, v) = state["case"], state["split"]
    weights = (state["q_weight"], state["k_weight"]) if case["norm"] else (None, None)
    if own:
        import paper_2607_00760_amd as mosaic
        return mosaic.qk_norm_rope(q, k, state["positions"], state["inv_freq"], *weights, eps=EPS, interleaved=case["interleaved"], v=v,
                                   axes=state["axes"])
    return _plain_axes(q, k, v, state["positions"], state["inv_freq"], *weights, case["interleaved"], state["axes"])


def _run_fill(state):
    cache, n = state["cache"], state["case"]["n"]
    cache["lens"].zero_()
    for k, v, counts in state["chunks"]:
        if own:
            state["handle"].append(k, v, counts)
        else:
            _plain_append(cache, k, v, counts)
    if own:
        k, v = state["handle"].read(n, 0, *state["out"])
    else:
        k, v = _plain_read(cache, n, torch.zeros_like(state["lens_dev"]), *state["out"])
    return {"k": k, "v": v, **{x: cache[x] for x in ("k_grid", "v_grid", "k_tail", "v_tail", "lens")}}


# ---------------------------------------------------------------- plain forms

def _plain_axes(q, k, v, positions, inv_freq, q_weight, k_weight, interleaved, axes):
    at = positions[torch.tensor(axes, device="cuda")].permute(1, 2, 0)     # [S][n][R / 2]: each pair's position
    angle = at.double() * inv_freq.double()
    cos, sin = (f(angle).float()[:, :, None] for f in (torch.cos, torch.sin))
    half = inv_freq.numel()

    def one(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
        if interleaved:
            a, b = y[..., 0: 2 * half: 2], y[..., 1: 2 * half: 2]
            z = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = y[..., :half], y[..., half: 2 * half]
            z = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        return torch.cat((z, y[..., 2 * half:]), -1).to(x.dtype)
    return one(q, q_weight), one(k, k_weight).transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous()


def _least(dtype):
    return 2.0 ** -100 if dtype == torch.bfloat16 else 2.0 ** -19


def _grid(x, dim):
    """Codes of 16-bit values x along rows of dimension dim, and the rows' scales and zeros."""
    dt, x = x.dtype, x.float()
    lo, hi = x.amin(dim, keepdim=True), x.amax(dim, keepdim=True)
    want = (hi * 0.5 - lo * 0.5) / torch.full_like(lo, 7.5)    # (a quotient of tensors: plain numbers divide through a reciprocal)
    scale = want.to(dt)
    down = (scale.view(torch.int16) - 1).view(dt)              # the value of the type below it
    scale = torch.where(scale.float() > want, down, scale).float().clamp_min(_least(dt))
    code = ((x * 0.5 - lo * 0.5) * (torch.full_like(scale, 2.0) / scale)).round()
    return code.to(torch.uint8), scale.to(dt).squeeze(dim), lo.to(dt).squeeze(dim)


def _pack(code):
    """Two codes a byte along the last dimension."""
    return code[..., 0::2] | code[..., 1::2] << 4


def _unpack(code):
    return torch.stack((code & 15, code >> 4), -1).flatten(-2)


def _plain_append(cache, k, v, counts):
    S, H, N, B, _ = cache["k"].shape
    L = cache["lens"][:, :1]                                   # [S][1], before the call
    f, n = L % B, counts[:, None]
    # the unfinished block and the new tokens, one after the other
    m = (k.shape[2] + B - 1) // B
    i = torch.arange(m * B + B, device="cuda")[None]
    at = torch.where(i < f, i, (i - f + B).clamp_max(B + k.shape[2] - 1)).long()[:, None, :, None].expand(S, H, -1, D)
    x = torch.cat((cache["k_tail"], k), 2).gather(2, at), torch.cat((cache["v_tail"].transpose(2, 3), v), 2).gather(2, at)
    done = (f + n) // B                                        # blocks that are whole now
    if m:
        xk, xv = (t[:, :, : m * B].reshape(S, H, m, B, D) for t in x)
        ck, sk, zk = _grid(xk, 3)
        cv, sv, zv = _grid(xv, 4)
        j = torch.arange(N, device="cuda")[None] - L // B      # which of these a block of the cache is
        new = ((j >= 0) & (j < done))[:, None]
        j = j.clamp(0, m - 1)[:, None].expand(S, H, N)
        for name, t in (("k", _pack(ck)), ("v", _pack(cv.transpose(3, 4))), ("k_grid", torch.stack((sk, zk), 3)),
                        ("v_grid", torch.stack((sv, zv), 3))):
            c = cache[name]
            fit = (S, H, N, 1, 1)
            c.copy_(torch.where(new.reshape(S, 1, N, 1, 1), t.gather(2, j.reshape(fit).expand_as(c)), c))
    rest = f + n - done * B
    t = torch.arange(B, device="cuda")[None]
    src = (done * B + t)[:, None, :, None].expand(S, H, B, D).long()
    left = ((t < rest) & ((done > 0) | (t >= f)))[:, None, :, None]
    cache["k_tail"].copy_(torch.where(left, x[0].gather(2, src), cache["k_tail"]))
    cache["v_tail"].copy_(torch.where(left, x[1].gather(2, src), cache["v_tail"].transpose(2, 3)).transpose(2, 3))
    cache["lens"] += n


def _fill8(cache, k, v, counts):
    """An empty 8-bit cache's codes and scales (for the inputs of `read`)."""
    B, top = cache["k"].shape[3], 448.0 if cache["k"].dtype == torch.float8_e4m3fn else 127.0
    nb, rest = divmod(int(counts.item()), B)
    for name, x in (("k", k), ("v", v)):
        if nb:
            b = x[:, :, : nb * B].float().unflatten(2, (nb, B))
            a = b.abs().amax((-1, -2)).clamp_min(2.0 ** -100)
            y = (b * (torch.full_like(a, top) / a)[..., None, None]).clamp(-top, top)
            y = (y if top == 448.0 else y.round()).to(cache[name].dtype)
            cache[name][:, :, :nb] = (y if name == "k" else y.view(torch.int8).transpose(3, 4).view(y.dtype))
            cache[name + "_scale"][:, :, :nb] = a / torch.full_like(a, top)
        tail = x[:, :, nb * B: nb * B + rest]
        if name == "k":
            cache["k_tail"][:, :, :rest] = tail
        else:
            cache["v_tail"][..., :rest] = tail.transpose(2, 3)
    cache["lens"].copy_(counts[:, None].expand_as(cache["lens"]))


def _values(cache):
    """What the codes stand for, in 32 bits: two [S][H][N B][D]."""
    if "k_grid" in cache:
        kg, vg = cache["k_grid"].float(), cache["v_grid"].float()
        k = kg[:, :, :, 1, None] + kg[:, :, :, 0, None] * _unpack(cache["k"]).float()
        v = vg[:, :, :, 1, :, None] + vg[:, :, :, 0, :, None] * _unpack(cache["v"]).transpose(3, 4).float()
    else:
        k = cache["k"].float() * cache["k_scale"][..., None, None]
        v = cache["v"].float().transpose(3, 4) * cache["v_scale"][..., None, None]
    return k.flatten(2, 3), v.flatten(2, 3)


def _plain_read(cache, n, starts, k_out, v_out):
    S, H, N, B, _ = cache["k"].shape
    L = cache["lens"][:, :1]
    t = starts[:, None] + torch.arange(n, device="cuda")[None]             # [S][n]
    whole, held = t < L // B * B, (t >= 0) & (t < L)
    for out, x, tail in zip((k_out, v_out), _values(cache), (cache["k_tail"], cache["v_tail"].transpose(2, 3))):
        at = t.clamp(0, N * B - 1).long()[:, None, :, None].expand(S, H, n, D)
        y = torch.where(whole[:, None, :, None], x.gather(2, at).to(out.dtype), tail.gather(2, at % B))
        out.copy_(torch.where(held[:, None, :, None], y, out))
    return k_out, v_out


def _plain_decode(cache, q, group):
    S, H, N, B, _ = cache["k"].shape
    k, v = _values(cache)
    q = q.float().view(S, H, group, D)
    L = cache["lens"][:, :1]
    seen = (torch.arange(N * B, device="cuda")[None] < L // B * B)[:, None, None]
    tail = (torch.arange(B, device="cuda")[None] < L % B)[:, None, None]
    z = (torch.matmul(q, k.transpose(2, 3)) * SCALE).masked_fill(~seen, -math.inf)
    zt = (torch.matmul(q, cache["k_tail"].float().transpose(2, 3)) * SCALE).masked_fill(~tail, -math.inf)
    top = torch.maximum(z.amax(-1, keepdim=True), zt.amax(-1, keepdim=True)).clamp_min(-3e38)
    p, pt = torch.exp(z - top), torch.exp(zt - top)
    total = p.sum(-1, keepdim=True) + pt.sum(-1, keepdim=True)
    out = torch.matmul(p, v) + torch.matmul(pt, torch.where(tail.transpose(2, 3), cache["v_tail"].float().transpose(2, 3), 0.0))
    return torch.where(total > 0, out / total, 0.0).flatten(1, 2)


def _plain_attend(cache, q, group, new_lens, causal, out):
    S, H, N, B, _ = cache["k"].shape
    n = q.shape[1]
    k, v = (torch.zeros((S, H, N * B, D), dtype=q.dtype, device="cuda") for _ in range(2))
    _plain_read(cache, N * B, torch.zeros_like(new_lens), k, v)
    L, m, i = cache["lens"][:, :1], new_lens[:, None], torch.arange(n, device="cuda")[None]
    last = L - m + i if causal else L - 1 + 0 * i              # [S][n]: the last token that a query attends
    hidden = (torch.arange(N * B, device="cuda") > last[..., None]).repeat_interleave(group, 1)[:, None]
    z = torch.matmul(q.float().view(S, n, H, group, D).transpose(1, 2).reshape(S, H, n * group, D), k.float().transpose(2, 3))
    z = z.mul_(SCALE).masked_fill_(hidden, -math.inf)
    p = z.sub_(z.amax(-1, keepdim=True).clamp_min(-3e38)).exp_()
    total = p.sum(-1, keepdim=True)
    y = torch.where(total > 0, torch.matmul(p, v.float()) / total, 0.0)
    y = y.view(S, H, n, group, D).transpose(1, 2).reshape(S, n, H * group, D).to(q.dtype)
    return out.copy_(torch.where((i < m)[:, :, None, None], y, out))


# ---------------------------------------------------------------- work

def _cache_bytes(case, L):
    """Codes, scales and zeros (or scales) of whole blocks of one head, its 16-bit tail: L tokens."""
    B = case["block"]
    one = D * B + 4 * D + 4 * B if _fmt(case) == "int4" else 2 * D * B + 8
    return L // B * one + L % B * 4 * D


def work(case):
    S, H, G, n = case["seqs"], case["hkv"], case["group"], case["n"]
    if case["op"] == "axes":
        rows = S * n * (H * G + 2 * H)
        return {"bytes": rows * 4 * D + S * n * 4 * case["num_axes"], "flops": rows * D * 8}
    lens = _lens(case)
    held = H * sum(_cache_bytes(case, L) for L in lens)
    if case["op"] == "fill":                                   # tokens in, the cache and the tokens out
        return {"bytes": 2 * H * sum(lens) * 4 * D + held, "flops": H * sum(lens) * 2 * D * 8}
    if case["op"] == "read":
        taken = [min(L, case["take"]) for L in lens]
        return {"bytes": H * sum(t * 4 * D + _cache_bytes(case, t) for t in taken), "flops": H * sum(taken) * 2 * D * 2}
    if case["op"] == "decode":
        return {"bytes": held + S * H * G * D * 6, "flops": 4 * H * G * D * sum(lens)}
    seen = sum(m * L - (m * (m - 1) // 2 if case["causal"] else 0) for m, L in zip(_new_lens(case), lens))
    return {"bytes": held + sum(_new_lens(case)) * H * G * D * 4, "flops": 4 * H * G * D * seen}


# ---------------------------------------------------------------- in 64 bits

def _f32(x):
    """64-bit values rounded to 32 bits."""
    return x.float().double()


def _stand_for(x, dt, dim):
    """Values of whole rows x along dim, in 64 bits: what their codes stand for; also the scales."""
    lo, hi = x.min(dim, keepdim=True).values, x.max(dim, keepdim=True).values
    want = _f32(_f32(hi / 2 - lo / 2) / 7.5)
    # the values of the type are whole multiples of these steps
    e = torch.floor(torch.log2(want.clamp(min=2.0 ** -140)))
    e = torch.where(torch.exp2(e) > want, e - 1, e)
    step = torch.exp2(e - 7) if dt == torch.bfloat16 else torch.exp2((e - 10).clamp(min=-24))
    scale = (torch.floor(want / step) * step).clamp(min=2.0 ** -100 if dt == torch.bfloat16 else 2.0 ** -19)
    code = torch.round(_f32(_f32(x / 2 - lo / 2) * _f32(2.0 / scale)))
    return lo + scale * code, scale, lo


def _stand_for8(x, fmt):
    top = 448.0 if fmt == "e4m3" else 127.0
    a = x.abs().flatten(1).max(1).values.clamp(min=2.0 ** -100)
    y = _f32(x * _f32(top / a)[:, None, None])
    if fmt == "e4m3":
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        y = (torch.round(y / step) * step).clamp(-448, 448)
    else:
        y = torch.round(y).clamp(-127, 127)
    return y * _f32(a / top)[:, None, None]


def _held(case, x, which):
    """One head's tokens x [n][D] as its cache holds them, in 64 bits."""
    B, dt = case["block"], _dtype(case)
    nb = x.shape[0] // B
    b = x[: nb * B].double().view(nb, B, D)
    if nb:
        b = _stand_for8(b, _fmt(case)) if _fmt(case) != "int4" else _stand_for(b, dt, 1 if which == "k" else 2)[0]
    return torch.cat((b.view(-1, D), x[nb * B:].double()))


def exact(case, seed):
    d = _inputs(case, seed)
    S, H, G, n = case["seqs"], case["hkv"], case["group"], case["n"]
    dt = _dtype(case)
    if case["op"] == "axes":
        if S * n * (G + 2) * H * D * 8 > 16 << 30:
            return None
        x, half, axes = d["qkv"].view(S, n, -1, D), case["rot"] // 2, _axes(case)

        def turned(x, w):
            y = x.double()
            if case["norm"]:
                y = y / torch.sqrt((y ** 2).sum(-1, keepdim=True) / D + EPS) * w.double()
            z = y.clone()
            for i in range(half):
                t = (d["positions"][axes[i]].double() * d["inv_freq"][i].double())[..., None]
                a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
                z[..., a] = y[..., a] * torch.cos(t) - y[..., b] * torch.sin(t)
                z[..., b] = y[..., a] * torch.sin(t) + y[..., b] * torch.cos(t)
            return z
        return (turned(x[:, :, : H * G], d["q_weight"]), turned(x[:, :, H * G: H * G + H], d["k_weight"]).transpose(1, 2).contiguous(),
                x[:, :, H * G + H:].double().transpose(1, 2).contiguous())
    lens = d["lens"]
    if case["op"] in ("fill", "read"):
        take = case["take"] if case["op"] == "read" else n
        o = {}
        for name in ("k", "v"):
            o[name] = torch.zeros((S, H, take, D), dtype=torch.float64, device="cuda")
            for s, L in enumerate(lens):
                a = d["starts"][s] if case["op"] == "read" else 0
                for h in range(H):
                    y = _held(case, d[name][s, h, :L], name)[a:]
                    o[name][s, h, : y.shape[0]] = y
        return o if case["op"] == "fill" else (o["k"], o["v"])
    if case["op"] == "decode":
        out = torch.zeros((S, H * G, D), dtype=torch.float64, device="cuda")
        for s, L in enumerate(lens):
            for h in range(H):
                at = slice(h * G, (h + 1) * G)
                k, v = _held(case, d["k"][s, h, :L], "k"), _held(case, d["v"][s, h, :L], "v")
                out[s, at] = torch.softmax(d["q"][s, at].double() @ k.T * SCALE, 1) @ v
        return out
    out = torch.zeros((S, case["new"], H * G, D), dtype=torch.float64, device="cuda")
    for s, (L, m) in enumerate(zip(lens, d["new_lens"])):
        for h in range(H):
            k, v = (_f32(_held(case, d[x][s, h, :L], x)).to(dt).double() for x in ("k", "v"))
            last = L - m + torch.arange(m, device="cuda") if case["causal"] else torch.full((m,), L - 1, device="cuda")
            hidden = torch.arange(L, device="cuda")[None] > last[:, None]
            for g in range(G):
                z = (d["q"][s, :m, h * G + g].double() @ k.T * SCALE).masked_fill(hidden, -math.inf)
                out[s, :m, h * G + g] = torch.softmax(z, 1) @ v
    return out
