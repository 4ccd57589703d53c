"""The entry points of the 4-bit cache, of the reading back of both caches and of
rotations with several axes, on the CPU: every refusal comes before anything is
enqueued, and every launch that fails is reported (over the recording HIP runtime
of tests/test_quant_args.py)."""
import ctypes as C

import pytest

from test_quant_args import CAPACITY, FAKE, HIP, INVALID, OK, UNSUPPORTED, _lib, lib, refused, three  # noqa: F401
from test_quant_args import cache as cache8

ARRAYS = ("k", "v", "k_grid", "v_grid", "k_tail", "v_tail", "lens", "arrivals", "refused")
LINES = ARRAYS[:6]                                             # those that vector loads read


def cache(**kw):
    c = _lib.MosaicNibbleCache(2, 8, 4, 128, 1, 64, 100, 0)
    for n in ARRAYS:
        setattr(c, n, FAKE)
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def append(lib, c, k=FAKE, v=FAKE, ks=three(8192, 1024, 128), vs=three(8192, 1024, 128), lens=None, n=8):
    return lib.mosaic_nibble_append(C.byref(c), k, v, ks, vs, lens, n, None)


def read(lib, c, k=FAKE, v=FAKE, ks=three(8192, 1024, 128), vs=three(8192, 1024, 128), starts=None, start=0, n=8):
    call = lib.mosaic_nibble_read if isinstance(c, _lib.MosaicNibbleCache) else lib.mosaic_quant_read
    return call(C.byref(c), k, v, ks, vs, starts, start, n, None)


def decode(lib, c, q=FAKE, out=FAKE, ws=FAKE, nbytes=1 << 40, scale=0.1):
    return lib.mosaic_nibble_decode_attention(C.byref(c), q, out, C.c_float(scale), ws, nbytes, None)


def attend(lib, c, q=FAKE, out=FAKE, qs=three(32768, 4096, 128), os=three(32768, 4096, 128), lens=None, n=8, ws=FAKE, nbytes=1 << 40,
           scale=0.1):
    return lib.mosaic_nibble_attend(C.byref(c), q, out, qs, os, lens, n, 1, C.c_float(scale), ws, nbytes, None)


def rope(lib, **kw):
    q, k = (_lib.MosaicRows(FAKE, FAKE, three(4096, 4096, 128), three(4096, 4096, 128)) for _ in range(2))
    a = dict(S=2, n=3, rot=128, ps=three(6, 3, 1), num=3, axes=bytes(i % 3 for i in range(64)))
    a.update(kw)
    return lib.mosaic_qk_norm_rope_axes(C.byref(q), C.byref(k), None, a["S"], a["n"], 32, 8, 128, 1, FAKE, FAKE, C.c_float(1e-6), FAKE, 4,
                                        a["ps"], FAKE, a["rot"], 0, a["num"], a["axes"], None)


CALLS = (append, read, decode, attend)


@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=64), UNSUPPORTED), (dict(block_len=16), UNSUPPORTED), (dict(block_len=128), UNSUPPORTED), (dict(dtype=2), INVALID),
    (dict(num_seqs=0), INVALID), (dict(num_kv_heads=0), INVALID), (dict(group_size=9), INVALID), (dict(group_size=0), INVALID),
    (dict(max_blocks=0), INVALID), (dict(num_seqs=40000), UNSUPPORTED), (dict(max_blocks=1 << 25), UNSUPPORTED), (dict(reserved=1), INVALID)])
def test_shapes_that_are_refused(lib, kw, status):  # noqa: F811
    c, n = cache(**kw), C.c_size_t()
    for call in CALLS:
        refused(lib, status, lambda: call(lib, c))
    refused(lib, status, lambda: lib.mosaic_nibble_workspace_bytes(C.byref(c), C.byref(n)))


def test_arrays_that_are_refused(lib):  # noqa: F811
    for name in ARRAYS:
        for bad in (None, FAKE + 2) + ((FAKE + 8,) if name in LINES else ()):
            for call in CALLS:
                refused(lib, INVALID, lambda: call(lib, cache(**{name: bad})))


def test_arguments_that_are_refused(lib):  # noqa: F811
    c, n = cache(), C.c_size_t()
    refused(lib, INVALID, lambda: lib.mosaic_nibble_workspace_bytes(C.byref(c), None))
    refused(lib, INVALID, lambda: lib.mosaic_nibble_workspace_bytes(None, C.byref(n)))
    assert lib.mosaic_nibble_workspace_bytes(C.byref(c), C.byref(n)) == OK
    rows = (dict(k=None), dict(v=None), dict(ks=None), dict(vs=None), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(ks=three(8192, 1024, 100)),
            dict(vs=three(8196, 1024, 128)), dict(n=-1))
    for kw in rows + (dict(lens=FAKE + 1),):
        refused(lib, INVALID, lambda: append(lib, c, **kw))
    for what in (c, cache8()):
        for kw in rows + (dict(starts=FAKE + 2), dict(ks=three(8192, 1024, 64)), dict(vs=three(0, 1024, 128)), dict(ks=three(8192, 0, 128))):
            refused(lib, INVALID, lambda: read(lib, what, **kw))
        lib.fake_reset(-1)
        assert read(lib, what, n=0) == OK and lib.fake_calls() == 0
        for start in (-5, 0, (1 << 31) - 1, -(1 << 31)):
            lib.fake_reset(-1)
            assert read(lib, what, start=start, n=(1 << 31) - 1) == OK and lib.fake_calls() == 1
    refused(lib, CAPACITY, lambda: append(lib, c, n=6401))
    refused(lib, UNSUPPORTED, lambda: append(lib, c, n=1 << 28, lens=FAKE))
    for kw in (dict(q=None), dict(out=None), dict(ws=None), dict(q=FAKE + 8), dict(out=FAKE + 8), dict(ws=FAKE + 16), dict(nbytes=n.value - 1),
               dict(scale=float("inf")), dict(scale=float("nan"))):
        refused(lib, INVALID, lambda: decode(lib, c, **kw))
        refused(lib, INVALID, lambda: attend(lib, c, **kw))
    for kw in (dict(qs=None), dict(os=None), dict(qs=three(32768, 4092, 128)), dict(os=three(32768, 4096, 4)), dict(os=three(32768, 4096, 64)),
               dict(os=three(32768, 0, 128)), dict(os=three(0, 4096, 128)), dict(n=-1), dict(lens=FAKE + 2)):
        refused(lib, INVALID, lambda: attend(lib, c, **kw))
    for big in ((1 << 27) + 1, 1 << 26):
        refused(lib, UNSUPPORTED, lambda: attend(lib, c, n=big))
    lib.fake_reset(-1)
    assert append(lib, c, n=0) == OK and attend(lib, c, n=0) == OK and lib.fake_calls() == 0
    # strides of a dimension of one row are not used, an input's rows may repeat
    one = cache(num_seqs=1)
    assert attend(lib, one, qs=three(1, 4096, 128), os=three(1, 4096, 128)) == OK and attend(lib, c, qs=three(0, 0, 0)) == OK


def test_launches_fit_a_grid(lib):  # noqa: F811
    """Threads along a launch's first dimension stay below 2^31."""
    g = (C.c_uint * 3)()
    for c, call in ((cache(num_seqs=1, num_kv_heads=1, max_blocks=1 << 23), lambda c: read(lib, c, n=(1 << 31) - 1)),
                    (cache(num_seqs=1, num_kv_heads=1, group_size=8), lambda c: attend(lib, c, n=1 << 24, lens=FAKE)),
                    (cache(num_seqs=8, num_kv_heads=8), lambda c: attend(lib, c, n=1 << 19)),
                    (cache(num_seqs=64512, num_kv_heads=1), lambda c: attend(lib, c, n=5))):
        lib.fake_reset(-1)
        status = call(c)
        if status != OK:
            assert status == UNSUPPORTED and lib.fake_calls() == 0
            continue
        for i in range(lib.fake_calls()):
            lib.fake_call_grid(i, g)
            assert g[0] * 512 < 1 << 32 and g[1] <= 65535 and g[2] == 1, list(g)


def test_axes_that_are_refused(lib):  # noqa: F811
    for kw in (dict(ps=None), dict(axes=None), dict(num=0), dict(num=256), dict(num=-1), dict(num=2), dict(axes=bytes(63) + b"\x03"),
               dict(axes=b"\xff" + bytes(63))):
        refused(lib, INVALID, lambda: rope(lib, **kw))
    for kw in (dict(rot=0), dict(rot=20), dict(rot=144), dict(n=1 << 22)):
        refused(lib, UNSUPPORTED, lambda: rope(lib, **kw))
    lib.fake_reset(-1)
    assert rope(lib) == OK and lib.fake_calls() == 1
    assert rope(lib, rot=32, axes=bytes([0, 1, 2] * 5 + [0])) == OK and rope(lib, num=255, axes=bytes([254] * 64)) == OK
    lib.fake_reset(-1)
    assert rope(lib, S=0) == OK and rope(lib, n=0) == OK and lib.fake_calls() == 0


@pytest.mark.parametrize("group", [1, 8])
@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("dtype", [0, 1])
def test_every_failed_launch_is_reported(lib, dtype, block, group):  # noqa: F811
    c = cache(block_len=block, dtype=dtype, group_size=group, max_blocks=400)
    calls = {"append": lambda: append(lib, c, n=1), "append_many": lambda: append(lib, c, n=5000), "decode": lambda: decode(lib, c),
             "read": lambda: read(lib, c), "few": lambda: attend(lib, c, n=2), "more": lambda: attend(lib, c, n=100 // group),
             "many": lambda: attend(lib, c, n=700), "rope": lambda: rope(lib)}
    for fmt in (0, 1):
        c8 = cache8(format=fmt, block_len=block, dtype=dtype)
        calls["read8", fmt] = lambda c8=c8: read(lib, c8)
    for name, call in calls.items():
        lib.fake_reset(-1)
        assert call() == OK, name
        n = lib.fake_calls()
        assert n, name
        for i in range(n):
            lib.fake_reset(i)
            assert call() == HIP and lib.mosaic_last_error(), (name, i)
