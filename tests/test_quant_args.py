"""The entry points of the 8-bit cache and of the norm-and-rotation pass on the
CPU: every refusal comes before anything is enqueued, and every launch that
fails is reported (over the recording HIP runtime)."""
import ctypes as C
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "hostsim"))

import build as hostsim_build  # noqa: E402  (tests/hostsim/build.py)
from paper_2607_00760_amd import _lib  # noqa: E402

OK, INVALID, UNSUPPORTED, CAPACITY, HIP = 0, -1, -2, -3, -5
FAKE = 0x100000
ARRAYS = ("k", "v", "k_scale", "v_scale", "bound_scale", "bounds", "k_tail", "v_tail", "lens", "arrivals", "refused")


@pytest.fixture(scope="module")
def lib():
    return _lib.bind_signatures(C.CDLL(hostsim_build.build_launches()))


def cache(**kw):
    c = _lib.MosaicQuantCache(2, 8, 4, 128, 1, 0, 32, 100)
    for n in ARRAYS:
        setattr(c, n, FAKE)
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def three(*s):
    return (C.c_int64 * 3)(*s)


def append(lib, c, k=FAKE, v=FAKE, ks=three(8192, 1024, 128), vs=three(8192, 1024, 128), lens=None, n=8):
    return lib.mosaic_quant_append(C.byref(c), k, v, ks, vs, lens, n, None)


def decode(lib, c, q=FAKE, out=FAKE, ws=FAKE, nbytes=1 << 40):
    return lib.mosaic_quant_decode_attention(C.byref(c), q, out, C.c_float(0.1), ws, nbytes, None)


def select(lib, c, q=FAKE, out=FAKE, ws=FAKE, nbytes=1 << 40, num=1, den=10, blocks=None):
    return lib.mosaic_quant_select_attention(C.byref(c), q, out, C.c_float(0.1), num, den, blocks, ws, nbytes, None)


def refused(lib, status, call):
    lib.fake_reset(-1)
    assert call() == status
    assert lib.mosaic_last_error() and lib.fake_calls() == 0


@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=64), UNSUPPORTED), (dict(block_len=16), UNSUPPORTED), (dict(block_len=0), UNSUPPORTED), (dict(dtype=2), INVALID),
    (dict(format=2), INVALID), (dict(num_seqs=0), INVALID), (dict(num_kv_heads=0), INVALID), (dict(group_size=9), INVALID),
    (dict(group_size=0), INVALID), (dict(max_blocks=0), INVALID), (dict(num_seqs=40000), UNSUPPORTED),
    (dict(max_blocks=1 << 26), UNSUPPORTED)])
def test_shapes_that_are_refused(lib, kw, status):
    c, n = cache(**kw), C.c_size_t()
    for call in (lambda: append(lib, c), lambda: decode(lib, c), lambda: select(lib, c),
                 lambda: lib.mosaic_quant_workspace_bytes(C.byref(c), C.byref(n))):
        refused(lib, status, call)


def test_arguments_that_are_refused(lib):
    c, n = cache(), C.c_size_t()
    for name in ARRAYS:
        bad = [cache(**{name: None}), cache(**{name: FAKE + 2})]
        for b in bad:
            for call in (lambda: append(lib, b), lambda: decode(lib, b), lambda: select(lib, b)):
                refused(lib, INVALID, call)
    refused(lib, INVALID, lambda: lib.mosaic_quant_workspace_bytes(C.byref(c), None))
    refused(lib, INVALID, lambda: lib.mosaic_quant_workspace_bytes(None, C.byref(n)))
    assert lib.mosaic_quant_workspace_bytes(C.byref(c), C.byref(n)) == OK and n.value >= 2 * 16 * 100 * 4
    for kw in (dict(k=None), dict(v=None), dict(ks=None), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(ks=three(8192, 1024, 100)),
               dict(vs=three(8196, 1024, 128)), dict(n=-1), dict(lens=FAKE + 1)):
        refused(lib, INVALID, lambda: append(lib, c, **kw))
    refused(lib, CAPACITY, lambda: append(lib, c, n=3201))
    refused(lib, UNSUPPORTED, lambda: append(lib, c, n=1 << 28, lens=FAKE))
    for call in (decode, select):
        for kw in (dict(q=None), dict(out=None), dict(ws=None), dict(q=FAKE + 8), dict(out=FAKE + 8), dict(ws=FAKE + 16),
                   dict(nbytes=n.value - 1)):
            refused(lib, INVALID, lambda: call(lib, c, **kw))
    for kw in (dict(num=0), dict(num=2, den=1), dict(den=0), dict(num=-1, den=-1), dict(blocks=FAKE + 1)):
        refused(lib, INVALID, lambda: select(lib, c, **kw))
    assert append(lib, c, n=0) == OK and lib.fake_calls() == 0


def rope(lib, **kw):
    q, k = (_lib.MosaicRows(FAKE, FAKE, three(4096, 4096, 128), three(4096, 4096, 128)) for _ in range(2))
    a = dict(q=q, k=k, v=None, S=2, n=3, hq=32, hkv=8, d=128, dt=1,
             qw=FAKE, kw=FAKE, eps=1e-6, pos=FAKE, pb=4, ps=(C.c_int64 * 2)(3, 1), inv=FAKE, rot=128)
    a.update(kw)
    ref = {x: C.byref(a[x]) if a[x] is not None else None for x in "qkv"}
    return lib.mosaic_qk_norm_rope(ref["q"], ref["k"], ref["v"], a["S"], a["n"], a["hq"], a["hkv"], a["d"], a["dt"], a["qw"], a["kw"],
                                   C.c_float(a["eps"]), a["pos"], a["pb"], a["ps"], a["inv"], a["rot"], 0, None)


def test_norm_rope_refusals(lib):
    def rows(**kw):
        r = _lib.MosaicRows(FAKE, FAKE, three(4096, 4096, 128), three(4096, 4096, 128))
        for x, y in kw.items():
            setattr(r, x, y)
        return r
    bad_rows = [rows(inp=None), rows(out=None), rows(inp=FAKE + 8), rows(out=FAKE + 4), rows(in_strides=three(4096, 4092, 128)),
                rows(out_strides=three(1, 4096, 128))]
    for r in bad_rows:
        for x in "qkv":
            refused(lib, INVALID, lambda: rope(lib, **{x: r}))
    for kw in (dict(q=None), dict(k=None), dict(pos=None), dict(ps=None), dict(inv=None), dict(dt=2), dict(S=-1), dict(n=-1), dict(hq=0),
               dict(hkv=0), dict(pb=2), dict(qw=None), dict(kw=None), dict(eps=-1.0), dict(eps=float("nan")), dict(pos=FAKE + 2),
               dict(pos=FAKE + 4, pb=8), dict(inv=FAKE + 2), dict(qw=FAKE + 8), dict(kw=FAKE + 2)):
        refused(lib, INVALID, lambda: rope(lib, **kw))
    for kw in (dict(d=64), dict(rot=0), dict(rot=20), dict(rot=144), dict(S=1 << 20, n=1 << 12), dict(n=1 << 22)):
        refused(lib, UNSUPPORTED, lambda: rope(lib, **kw))
    lib.fake_reset(-1)
    assert rope(lib, S=0) == OK and rope(lib, n=0) == OK and lib.fake_calls() == 0
    assert rope(lib, qw=None, kw=None) == OK and lib.fake_calls() == 1


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("dtype", [0, 1])
def test_every_failed_launch_is_reported(lib, fmt, block, dtype):
    c = cache(format=fmt, block_len=block, dtype=dtype)
    calls = {"append": lambda: append(lib, c, n=1), "append_many": lambda: append(lib, c, n=500), "decode": lambda: decode(lib, c),
             "select": lambda: select(lib, c), "select_long": lambda: select(lib, cache(max_blocks=40000, format=fmt, block_len=block)),
             "rope": lambda: rope(lib, dt=dtype)}
    for name, call in calls.items():
        lib.fake_reset(-1)
        assert call() == OK
        n = lib.fake_calls()
        assert n
        for i in range(n):
            lib.fake_reset(i)
            assert call() == HIP and lib.mosaic_last_error(), (name, i)
