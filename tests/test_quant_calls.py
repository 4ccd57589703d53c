"""Further calls of the operators around the 8-bit cache on the CPU: what is
refused before anything is enqueued, and what is not (over the recording HIP
runtime of tests/test_quant_args.py)."""
import ctypes as C

import pytest

from test_quant_args import FAKE, INVALID, OK, _lib, append, cache, lib, refused, rope, three  # noqa: F401


def rows(ins=(4096, 4096, 128), outs=(4096, 4096, 128)):
    return _lib.MosaicRows(FAKE, FAKE, three(*ins), three(*outs))


@pytest.mark.parametrize("outs", [(0, 4096, 128), (4096, 0, 128), (4096, 4096, 0), (4096, 4096, 64), (4096, 4096, -120), (8, 4096, 128)])
def test_outputs_whose_rows_overlap(lib, outs):  # noqa: F811
    """An expanded output would have its rows written by several workgroups."""
    for x in "qkv":
        refused(lib, INVALID, lambda: rope(lib, **{x: rows(outs=outs)}))
        lib.fake_reset(-1)                                     # an input may repeat its rows
        assert rope(lib, **{x: rows(ins=outs)}) == OK and lib.fake_calls() == 1


def test_outputs_of_one_row_along_a_dimension(lib):  # noqa: F811
    for kw, outs in ((dict(S=1), (0, 4096, 128)), (dict(n=1), (4096, 0, 128)), (dict(hkv=1), (4096, 128, 0)), (dict(), (4096, 512, -128))):
        lib.fake_reset(-1)
        assert rope(lib, k=rows(outs=outs), **kw) == OK and lib.fake_calls() == 1


def test_strides_along_one_row(lib):  # noqa: F811
    """A dimension of one row has no alignment: its stride is not used."""
    for kw, st in ((dict(S=1), (1, 4096, 128)), (dict(n=1), (4096, 1, 128)), (dict(hkv=1), (4096, 4096, 1))):
        lib.fake_reset(-1)
        assert rope(lib, k=rows(st, st), v=rows(st, st), **kw) == OK and lib.fake_calls() == 1
        refused(lib, INVALID, lambda: rope(lib, k=rows(ins=st)))
    for c, n, st in ((cache(num_seqs=1), 8, (1, 1024, 128)), (cache(num_kv_heads=1), 8, (8192, 1, 128)), (cache(), 1, (8192, 1024, 1))):
        lib.fake_reset(-1)
        assert append(lib, c, ks=three(*st), vs=three(*st), n=n) == OK and lib.fake_calls() == 1
        refused(lib, INVALID, lambda: append(lib, cache(), ks=three(*st)))


@pytest.mark.parametrize("hq,hkv", [(65535 * 16, 1), (1 << 20, 8), (1 << 20, 1 << 20), (32, 1 << 20)])
def test_many_heads_fit_a_grid(lib, hq, hkv):  # noqa: F811
    """A grid's second dimension holds 65535 workgroups."""
    lib.fake_reset(-1)
    assert rope(lib, hq=hq, hkv=hkv, v=rows(), n=1) == OK and lib.fake_calls() == 1
    g = (C.c_uint * 3)()
    lib.fake_call_grid(0, g)
    assert g[0] == 2 and g[1] <= 65535 and g[2] == 1
