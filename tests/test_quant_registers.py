"""The kernels of the 8-bit cache and of the norm-and-rotation pass keep their
values in registers (read from the code objects' own metadata)."""
import os
import re

import pytest

from test_kernel_registers import READELF, kernels


@pytest.mark.skipif(not os.path.exists(READELF), reason="needs ROCm's llvm-readelf")
def test_no_spills():
    found = {n: v for n, v in kernels().items() if re.search(r"k_(quant_(attn|append|score|topk|lens)|norm_rope)(I|E)", n)}
    for name, n in (("k_quant_attnI", 16), ("k_quant_appendI", 8), ("k_quant_scoreI", 2), ("k_quant_topkI", 4), ("k_norm_ropeI", 4)):
        assert sum(name in x for x in found) >= n, (name, sorted(found))
    assert not {n: v for n, v in found.items() if v != (0, 0)}


@pytest.mark.skipif(not os.path.exists(READELF), reason="needs ROCm's llvm-readelf")
def test_no_spills_in_the_selection_of_small_caches():
    found = {n: v for n, v in kernels().items() if re.search(r"k_quant_pickI", n)}
    assert len(found) == 2 and not {n: v for n, v in found.items() if v != (0, 0)}, found
