"""Builds and calls attention_probe.cpp: which kernels the host layer of the
attention-side operators would launch for a call of the C ABI (CPU only)."""
from __future__ import annotations

import ctypes
import functools
import os
import subprocess
import tempfile

from paper_2305_17190_amd import attention as att
from paper_2305_17190_amd import build

FORMS = {1: "whole", 2: "scores", 3: "values", 4: "join", 5: "tile scores", 6: "tile values", 7: "heads", 8: "gradient"}
MOST = 64


class Launch(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int64) for name in ("form", "bf16", "lanes", "rows", "fine", "units", "first_unit",
                                                    "splits", "split_keys", "threads")]

    @property
    def name(self) -> str:
        return FORMS[self.form]


@functools.lru_cache(maxsize=None)
def library() -> ctypes.CDLL:
    here = os.path.dirname(os.path.abspath(__file__))
    with tempfile.TemporaryDirectory() as tmp:
        so = os.path.join(tmp, "attention_probe.so")
        rocm = os.path.join(os.path.dirname(os.path.dirname(build.hipcc())), "include")
        subprocess.run(["g++", "-std=c++17", "-O1", "-w", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__",
                        "-isystem", rocm, "-I", build.INCLUDE, "-I", build.CSRC,
                        os.path.join(here, "attention_probe.cpp"), "-o", so], check=True)
        lib = ctypes.CDLL(so)
    i32, vp = ctypes.c_int32, ctypes.c_void_p
    for name in att.EXPORTS:
        if not name.endswith("_workspace_size"):
            getattr(lib, name).argtypes = [ctypes.c_char_p, vp]
        getattr(lib, name).restype = i32
    lib.pam_paged_attention_workspace_size.argtypes = [i32] * 7 + [ctypes.POINTER(ctypes.c_size_t)]
    lib.probe_take.argtypes = [ctypes.POINTER(Launch)]
    lib.probe_take.restype = i32
    lib.probe_error.restype = ctypes.c_char_p
    return lib


def take():
    """The launches since the last call, the first MOST of them."""
    out = (Launch * MOST)()
    count = library().probe_take(out)
    return list(out[:min(count, MOST)])


PTR = 1 << 20   # stands for every device address


class Heads(ctypes.Structure):
    _fields_ = [("stride_token", ctypes.c_int64), ("stride_head", ctypes.c_int64), ("heads", ctypes.c_int32),
                ("type", ctypes.c_int32)]


class Cache(ctypes.Structure):
    _fields_ = [("stride_page", ctypes.c_int64), ("stride_slot", ctypes.c_int64), ("stride_head", ctypes.c_int64),
                ("pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("type", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class Attention(ctypes.Structure):
    _fields_ = ([(name, ctypes.c_void_p) for name in ("q", "k_cache", "v_cache", "q_starts", "kv_lens", "table", "out",
                                                      "workspace")]
                + [("q_heads", Heads), ("out_heads", Heads), ("k_cache_layout", Cache), ("v_cache_layout", Cache),
                   ("table_stride", ctypes.c_int64), ("tokens", ctypes.c_int64)]
                + [(name, ctypes.c_int32) for name in ("d", "batch", "table_width", "causal", "window")]
                + [("scale", ctypes.c_float), ("max_q", ctypes.c_int32), ("max_kv", ctypes.c_int32),
                   ("workspace_bytes", ctypes.c_int64)])


def workspace(d, heads, group, bf16, batch, max_q, max_kv) -> int:
    need = ctypes.c_size_t()
    assert library().pam_paged_attention_workspace_size(d, heads * group, heads, int(bf16), batch, max_q, max_kv,
                                                        ctypes.byref(need)) == 0
    return need.value


def attention(d, heads, group, bf16, batch, max_q, max_kv):
    """(status, launches) of an attention call over dense operands."""
    q = Heads(heads * group * d, d, heads * group, 0)
    cache = Cache(16 * heads * d, heads * d, d, 10, 16, heads, int(bf16), 0)
    width = -(-max_kv // 16)
    args = Attention(PTR, PTR, PTR, PTR if max_q > 1 else None, PTR, PTR, PTR, PTR, q, q, cache, cache, width,
                     batch * max_q, d, batch, width, 1, 0, 1.0, max_q, max_kv, 1 << 60)
    take()
    status = library().pam_paged_attention(bytes(args), None)
    return status, take()


def form(d, heads, group, bf16, batch, max_q, max_kv):
    """("whole", "split" or "tiles"; fine; rows a unit; lanes a key) of a call
    with these bounds."""
    status, launches = attention(d, heads, group, bf16, batch, max_q, max_kv)
    assert status == 0, library().probe_error()
    first = launches[0]
    return {"whole": "whole", "scores": "split", "tile scores": "tiles"}[first.name], bool(first.fine), first.rows, first.lanes
