"""Build libmosaic.so (HIP, gfx950) in-tree with hipcc.

All HIP sources are compiled with fp contraction off (every fused multiply-add
in the kernels is an explicit fmaf) and with the packed-fp32 instructions
disabled.  A HIP error that is dropped without saying so does not compile.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmosaic.so")
ARCH = os.environ.get("MOSAIC_OFFLOAD_ARCH", "gfx950")
SOURCES = ["api.hip", "attn_bf16_g4.hip", "attn_bf16_g8.hip", "attn_fp16_g4.hip", "attn_fp16_g8.hip", "compress.hip",
           "decode.hip", "dense.hip", "encode.hip", "norm_rope.hip", "quant4_append.hip", "quant4_attn.hip", "quant4_chunk.hip", "quant_api.hip",
           "quant_append.hip", "quant_attn_e4m3.hip", "quant_attn_int8.hip", "quant_read.hip", "quant_select.hip", "rotation.hip", "score.hip"]
FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unused-variable", "-Werror=unused-value",
]


def _hipcc():
    for c in ("/opt/rocm/bin/hipcc", "hipcc"):
        if os.path.exists(c) or c == "hipcc":
            return c


def build(verbose: bool = False) -> str:
    """Compile every HIP source and link the shared library (always rebuilds)."""
    hipcc = _hipcc()
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(objdir, os.path.splitext(src)[0] + ".o")
        cmd = [hipcc, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{r.stderr}")
        if verbose and r.stderr.strip():
            sys.stderr.write(r.stderr)
        return obj

    with cf.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB + ".tmp%d" % os.getpid()
    r = subprocess.run([hipcc, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
