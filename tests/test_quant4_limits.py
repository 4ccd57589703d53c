"""Limits of the 4-bit cache's entry points, on the CPU (over the recording HIP
runtime of tests/test_quant_args.py)."""
import ctypes as C

import pytest

from test_quant4_args import attend, cache, decode
from test_quant_args import FAKE, INVALID, OK, lib, refused  # noqa: F401


@pytest.mark.parametrize("scale,fits", [(2.0 ** 127, True), (-2.0 ** 127, True), (0.0, True), (1e-45, True), (2.0 ** 127 * (1 + 2.0 ** -23), False),
                                        (-3.4e38, False), (float("inf"), False), (float("nan"), False)])
def test_softmax_scales(lib, scale, fits):  # noqa: F811
    for call in (decode, attend):
        if fits:
            lib.fake_reset(-1)
            assert call(lib, cache(), scale=scale) == OK and lib.fake_calls()
        else:
            refused(lib, INVALID, lambda: call(lib, cache(), scale=scale))


@pytest.mark.parametrize("S,H,block,N", [(256, 1, 64, 100), (300, 8, 32, 100), (255, 1, 64, 100), (1, 1, 64, 4), (1, 1, 64, 5), (2, 8, 32, 8),
                                         (2, 8, 32, 9), (7, 5, 32, 1)])
def test_workspace_of_shares(lib, S, H, block, N):  # noqa: F811
    """The workspace has room for the shares of several tokens where a launch shares
    (and is followed by the launch that joins them), and nowhere else."""
    n = C.c_size_t()
    most = []
    for G in (1, 8):
        c = cache(num_seqs=S, num_kv_heads=H, block_len=block, max_blocks=N, group_size=G)
        assert lib.mosaic_nibble_workspace_bytes(C.byref(c), C.byref(n)) == OK
        for m in (1, 2, 4, 5, 16, 17, 32, 33, 100, 128, 129, 300, 2000):
            lib.fake_reset(-1)
            assert attend(lib, c, n=m, lens=FAKE, nbytes=n.value) == OK
            most.append(lib.fake_calls())
    runs = (512 - S * H if S * H <= 256 else 1024) + S * H
    single = -(-((1 << 19) + runs * 8 * 130 * 4) // 256) * 256
    shares = n.value - single
    assert shares in (0, 256 * (256 * 132 * 4 + 8)) and max(most) == (2 if shares else 1)
