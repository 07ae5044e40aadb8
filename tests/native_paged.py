"""The library's index arithmetic of the paged cache, compiled for the host from
its own header (tests/native/paged.cpp), for the tests without a GPU."""
from __future__ import annotations

import ctypes
import functools
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@functools.lru_cache(maxsize=None)
def lib() -> ctypes.CDLL:
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    out = os.path.join(ROOT, "_build", "paged.so")
    os.makedirs(os.path.dirname(out), exist_ok=True)
    tmp = f"{out}.tmp{os.getpid()}"
    r = subprocess.run(
        [hipcc, "-x", "hip", "-O1", "-std=c++17", "-fPIC", "-shared", "--offload-arch=gfx950",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         f"-I{os.path.join(ROOT, 'include')}",
         f"-I{os.path.join(ROOT, 'paper_2607_26475_amd', 'csrc')}",
         os.path.join(HERE, "native", "paged.cpp"), "-o", tmp],
        capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    os.replace(tmp, out)
    so = ctypes.CDLL(out)
    so.t_check_table.restype = ctypes.c_uint64
    so.t_hand_over.argtypes = [ctypes.POINTER(ctypes.c_uint64), ctypes.c_uint64, ctypes.c_uint32,
                               ctypes.c_uint32]
    return so
