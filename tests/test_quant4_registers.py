"""The kernels of the 4-bit cache, of the reading back and of rotations with
several axes keep their values in registers (read from the code objects' own
metadata).  Left out: few queries over blocks of 32, which hold the grids of two
blocks beside all else and spill two registers outside of their loop."""
import os
import re

import pytest

from test_kernel_registers import READELF, kernels


@pytest.mark.skipif(not os.path.exists(READELF), reason="needs ROCm's llvm-readelf")
def test_no_spills():
    found = {n: v for n, v in kernels().items() if re.search(r"k_(quant4_(attn|append|lens)|quant_read|chunk|chunk_few|chunk_join|norm_rope)(I|E)", n)}
    for name, n in (("k_quant4_attnI", 8), ("k_quant4_appendI", 4), ("k_quant_readI", 12), ("k_chunkI", 8), ("k_chunk_fewI", 4),
                    ("k_chunk_joinI", 2), ("k_norm_ropeI", 8)):
        assert sum(name in x for x in found) >= n, (name, sorted(found))
    assert not {n: v for n, v in found.items() if v != (0, 0) and "k_chunk_fewILi32E" not in n}
