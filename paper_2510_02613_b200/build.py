"""Builds libemoe.so (host planner + C ABI + sm_100a kernels) in-tree with nvcc."""
from __future__ import annotations

import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
SOURCES = ["planner.cpp", "capi.cpp", "vmm.cpp", "placement.cpp", "cache.cpp", "validate.cpp", "serve.cpp", "kernels.cu", "kv_cache.cu", "kv_extend.cu", "attend.cu", "attend_prefix.cu", "attend_masked.cu", "attend_masked_few.cu", "attend_masked_tensor.cu", "moe.cu"]
HEADERS = ["planner.h", "kernels.h", "internal.h", "serve.h", "convert.cuh", "attend_item.cuh", "attend_masked.cuh", "tensor.cuh", os.path.join("..", "..", "include", "emoe.h")]
OUT = os.path.join(HERE, "libemoe.so")


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: libemoe.so cannot be built")


def have_nvcc() -> bool:
    try:
        _nvcc()
        return True
    except RuntimeError:
        return False


def is_stale() -> bool:
    if not os.path.exists(OUT):
        return True
    t = os.path.getmtime(OUT)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not is_stale():
        return OUT
    tmp = OUT + ".%d.tmp" % os.getpid()
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
           "-shared", "-Xcompiler", "-fPIC,-Wall", "-x", "cu", "-t", "0",
           "-o", tmp] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    subprocess.check_call(cmd)
    os.replace(tmp, OUT)
    return OUT


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
