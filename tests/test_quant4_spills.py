"""How many values of the 4-bit cache's kernels leave the registers: none, but six
(28 bytes of scratch, outside of its loop) of few bf16 queries over blocks of 32,
which hold the grids of two blocks beside all else.  Read from the code objects'
own metadata."""
import os
import re

import pytest

from test_kernel_registers import READELF, kernels


@pytest.mark.skipif(not os.path.exists(READELF), reason="needs ROCm's llvm-readelf")
def test_spills():
    found = {n: v for n, v in kernels().items() if re.search(r"k_(quant4_\w+?|quant_read|chunk|chunk_few|chunk_join)(I|E)", n)}
    few = [v for n, v in found.items() if "k_chunk_fewILi32ELi1E" in n]
    assert len(found) >= 39 and len(few) == 1 and few[0][0] <= 6 and few[0][1] <= 28, few
    assert not {n: v for n, v in found.items() if v != (0, 0) and "k_chunk_fewILi32ELi1E" not in n}
