"""Build the sm_100a shared library in-tree with nvcc."""
from __future__ import annotations

import os
import shutil
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libpcr_b200.so")
SOURCES = ["pcr_lib.cu", "pcr_tokens.cu", "pcr_decay.cu", "pcr_decay_tiles.cu", "pcr_bias.cu"]
HEADERS = ["pcr_types.h", "pcr_entropy.cuh", "pcr_long.cuh", "pcr_pixels.cuh", "pcr_refine.cuh", "pcr_walks.h", "pcr_sequential.cuh", "pcr_msssim.cuh",
           "pcr_bias.cuh", "pcr_decay.cuh", "pcr_decay_tiles.cuh", "pcr_decay_tiles.h", "pcr_heads.cuh", "pcr_launches.h", "pcr_patches.cuh", "pcr_spans.h"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA library cannot be built")


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.join(os.path.dirname(_HERE), "include", "pcr.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """nvcc -> libpcr_b200.so next to this file (sm_100a only)."""
    if not force and not stale():
        return LIB
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-t", "0",
           "-shared", "-Xcompiler", "-fPIC", "-o", tmp]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += os.environ.get("PCR_NVCC_FLAGS", "").split()
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
