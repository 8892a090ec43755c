"""Build step for the HIP library libpam.so (gfx950 only).

    python -m paper_2305_17190_amd.build

compiles csrc/*.hip and csrc/*.cpp with hipcc into paper_2305_17190_amd/libpam.so,
one object per source (the matrix product kernels in PARTS of their source),
several at a time; and csrc/python/pack.cpp with g++ into _pack.so, the part of
the Python binding that reads torch tensors.
"""
from __future__ import annotations

import concurrent.futures
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libpam.so")
PACK = os.path.join(PKG, "_pack.so")

# Device code: gfx950 only; float32 denormals flushed (the GEMM relies on the
# accumulate treating denormal encodings as zero); no packed-fp32 VALU ops.
DEVICE_FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fgpu-flush-denormals-to-zero",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def hipcc() -> str:
    path = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(path):
        raise RuntimeError("hipcc not found; the PAM library needs ROCm's hipcc")
    return path


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".hip", ".cpp")))


# Sources compiled in parts, one object each (their count of parts).
PARTS = {"pam_gemm_dma.hip": 6}


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed to build the PAM library")


def _build_pack(verbose: bool) -> None:
    """_pack.so, against the headers and libraries of the installed torch (found
    without importing it)."""
    torch = importlib.util.find_spec("torch").submodule_search_locations[0]
    includes = [os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include"),
                os.path.join(os.path.dirname(os.path.dirname(hipcc())), "include")]
    tmp = f"{PACK}.{os.getpid()}.tmp"
    _run(["g++", "-O2", "-std=c++17", "-w", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
          "-I", sysconfig.get_paths()["include"], *(x for path in includes for x in ("-isystem", path)),
          os.path.join(CSRC, "python", "pack.cpp"), "-o", tmp, "-L", os.path.join(torch, "lib"), "-ltorch_python",
          "-ltorch_cpu", "-ltorch", "-lc10"], verbose)
    os.replace(tmp, PACK)


def build(verbose: bool = False, extra_flags=()) -> str:
    flags = [hipcc(), *DEVICE_FLAGS, *extra_flags, "-fPIC"]
    with tempfile.TemporaryDirectory() as tmpdir:
        jobs = []
        for src in sources():
            name = os.path.basename(src)
            for part in range(PARTS.get(name, 1)):
                obj = os.path.join(tmpdir, f"{name}.{part}.o")
                define = [f"-DPAM_GEMM_PART={part}"] if name in PARTS else []
                jobs.append(([*flags, *define, "-I", INCLUDE, "-I", CSRC, "-c", src, "-o", obj], obj))
        with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
            pack = pool.submit(_build_pack, verbose)
            for done in [pool.submit(_run, cmd, verbose) for cmd, _ in jobs] + [pack]:
                done.result()
        tmp = f"{LIB}.{os.getpid()}.tmp"   # per process: concurrent builds never see a partial file
        _run([*flags, "-shared", *(obj for _, obj in jobs), "-o", tmp, "-lhsa-runtime64"], verbose)
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
