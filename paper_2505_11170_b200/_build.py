"""Builds the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
CSRC = os.path.join(_PKG, "csrc")
INCLUDE = os.path.join(_ROOT, "include")
LIB_PATH = os.path.join(_PKG, "libgws.so")
# Two translation units: the sampling pass (gws_api.cu) and the activation operators (gws_block.cu).
_UNITS = {
    "gws_api.cu": ["gws_kernels.cuh", "gws_math.cuh", "gws_gemm.cuh", "gws_probe.cuh", "gws_compare.cuh", "gws_gemm_cluster.cuh", "gws_gemm_wide.cuh",
                   "gws_train.cuh", "gws_internal.h"],
    "gws_block.cu": ["gws_tc.cuh", "gws_act8.cuh", "gws_internal.h"],
}
SOURCES = [os.path.join(CSRC, name) for name in _UNITS]
HEADERS = sorted({os.path.join(CSRC, h) for hs in _UNITS.values() for h in hs}) + [os.path.join(INCLUDE, "gws.h")]

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-I" + INCLUDE, "-I" + CSRC]
# -fmad=false: the add-then-cast path must round the multiply and the add separately.
_UNIT_FLAGS = {"gws_api.cu": ["-fmad=false"], "gws_block.cu": []}


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


CHECK_LIB_PATH = os.path.join(_PKG, "libgws_check.so")   # the self-checking variant (-DGWS_SELF_CHECK)


def is_stale(path: str = LIB_PATH) -> bool:
    if not os.path.exists(path):
        return True
    built = os.path.getmtime(path)
    return any(os.path.getmtime(p) > built for p in SOURCES + HEADERS)


def _unit_is_stale(obj: str, unit: str) -> bool:
    if not os.path.exists(obj):
        return True
    built = os.path.getmtime(obj)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > built for f in [unit, *_UNITS[unit]]) or \
        os.path.getmtime(os.path.join(INCLUDE, "gws.h")) > built


def build(force: bool = False, verbose: bool = False, self_check: bool = False) -> str:
    """Compile ``libgws.so`` (or the self-checking ``libgws_check.so``) next to the package if it is missing
    or older than its sources.  Each translation unit is compiled to an object of its own, side by side."""
    path = CHECK_LIB_PATH if self_check else LIB_PATH
    if force or is_stale(path):
        objects = os.path.join(_PKG, "_build")
        os.makedirs(objects, exist_ok=True)
        extra = [*(["-DGWS_SELF_CHECK"] if self_check else []), *(["-Xptxas", "-v"] if verbose else [])]

        def compile_unit(unit: str) -> str:
            obj = os.path.join(objects, os.path.splitext(unit)[0] + ("_check.o" if self_check else ".o"))
            if force or _unit_is_stale(obj, unit):
                tmp = obj + ".tmp.%d" % os.getpid()
                subprocess.run([_nvcc(), *NVCC_FLAGS, *_UNIT_FLAGS[unit], *extra, "-c", "-o", tmp, os.path.join(CSRC, unit)], check=True)
                os.replace(tmp, obj)
            return obj

        with ThreadPoolExecutor(max_workers=len(_UNITS)) as pool:
            built = list(pool.map(compile_unit, _UNITS))
        tmp = path + ".tmp.%d" % os.getpid()
        subprocess.run([_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-Xcompiler", "-fPIC", "-o", tmp, *built], check=True)
        os.replace(tmp, path)
    return path


if __name__ == "__main__":
    print(build(force=True, verbose=True))
