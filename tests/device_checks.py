"""Builds and loads device_checks.cu, parts of the kernels by themselves.  Test infrastructure."""
from __future__ import annotations

import ctypes
import os
import subprocess

from paper_2510_02613_b200 import build

HERE = os.path.dirname(os.path.abspath(__file__))


def load(folder) -> ctypes.CDLL:
    out = os.path.join(str(folder), "device_checks.so")
    subprocess.check_call([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo", "-shared", "-Xcompiler", "-fPIC,-Wall",
                           "-o", out, os.path.join(HERE, "device_checks.cu")])
    lib = ctypes.CDLL(out)
    vp, i32, u64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64
    lib.check_order.argtypes, lib.check_wait.argtypes = [vp, i32, i32, i32, i32, i32, vp], [i32, u64, u64, vp, vp]
    return lib
