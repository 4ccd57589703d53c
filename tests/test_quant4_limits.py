"""Limits of the 4-bit cache's entry points, on the CPU (over the recording HIP
runtime of tests/test_quant_args.py)."""
import pytest

from test_quant4_args import attend, cache, decode
from test_quant_args import INVALID, OK, lib, refused  # noqa: F401


@pytest.mark.parametrize("scale,fits", [(2.0 ** 127, True), (-2.0 ** 127, True), (0.0, True), (1e-45, True), (2.0 ** 127 * (1 + 2.0 ** -23), False),
                                        (-3.4e38, False), (float("inf"), False), (float("nan"), False)])
def test_softmax_scales(lib, scale, fits):  # noqa: F811
    for call in (decode, attend):
        if fits:
            lib.fake_reset(-1)
            assert call(lib, cache(), scale=scale) == OK and lib.fake_calls()
        else:
            refused(lib, INVALID, lambda: call(lib, cache(), scale=scale))
