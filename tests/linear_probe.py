"""Builds and calls linear_probe.cpp and dispatch_probe.cpp: which kernels the
library's host layer would launch for a linear layer (CPU only)."""
from __future__ import annotations

import ctypes
import functools
import os
import struct
import subprocess
import tempfile

import paper_2305_17190_amd as pam
from dispatch_probe import Launch
from paper_2305_17190_amd import build


@functools.lru_cache(maxsize=None)
def library() -> ctypes.CDLL:
    here = os.path.dirname(os.path.abspath(__file__))
    with tempfile.TemporaryDirectory() as tmp:
        so = os.path.join(tmp, "linear_probe.so")
        rocm = os.path.join(os.path.dirname(os.path.dirname(build.hipcc())), "include")
        subprocess.run(["g++", "-std=c++17", "-O1", "-w", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__",
                        "-isystem", rocm, "-I", build.INCLUDE, "-I", build.CSRC, os.path.join(here, "linear_probe.cpp"),
                        os.path.join(here, "dispatch_probe.cpp"), "-o", so], check=True)
        lib = ctypes.CDLL(so)
    i64, vp, psz = ctypes.c_int64, ctypes.c_void_p, ctypes.POINTER(ctypes.c_size_t)
    lib.pam_linear.argtypes = [ctypes.c_char_p, vp]
    lib.pam_linear_workspace_size.argtypes = [i64, i64, i64, psz]
    lib.pam_gemm_workspace_size.argtypes = [i64, i64, i64, i64, psz]
    lib.pam_last_error.restype = ctypes.c_char_p
    lib.probe_take.argtypes = [ctypes.POINTER(Launch)]
    return lib


def workspace(m, n, k):
    """(bytes of the layer, bytes of the product alone)."""
    need = [ctypes.c_size_t(), ctypes.c_size_t()]
    assert library().pam_linear_workspace_size(m, n, k, ctypes.byref(need[0])) == 0
    assert library().pam_gemm_workspace_size(m, n, k, 1, ctypes.byref(need[1])) == 0
    return need[0].value, need[1].value


def linear(m, k, n, bf16=False, ldy=None):
    """The launches of a layer of dense operands with bias and residual, at most
    the first eight, and their count."""
    at = [(i + 1) << 50 for i in range(7)]      # stand-in addresses, far apart
    ldy = ldy or max(n, 1)
    args = struct.pack("=7q9q4i", *at[:4], at[4], 0, at[6], m, n, k, max(k, 1), max(k, 1), max(n, 1), ldy, 0,
                       workspace(m, n, k)[0], int(bf16), 0, 2, 23)
    status = library().pam_linear(args, None)
    assert status == 0, library().pam_last_error()
    out = (Launch * 8)()
    count = library().probe_take(out)
    return list(out[:min(count, 8)]), count
