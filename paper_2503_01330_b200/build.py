"""Compiles the CUDA library in-tree for sm_100a with nvcc (no GPU needed: nvcc cross-compiles)."""
from __future__ import annotations

import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libwkv.so")
OBJ_DIR = os.path.join(_HERE, "_build")
HEADER = os.path.join("..", "..", "include", "wkv.h")
PAGED = ["wkv_ptx.cuh", "wkv_paged.cuh", "wkv_paged_host.cuh", HEADER]
# source -> what it includes; each is compiled to an object of its own, rebuilt when one of them is newer
UNITS = {
    "wkv_api.cu": ["wkv_ptx.cuh", "wkv_kernels.cuh", "wkv_prefill.cuh", "wkv_block.cuh", HEADER],
    "wkv_paged_api.cu": [*PAGED, "wkv_paged_decode.cuh", "wkv_paged_evict.cuh", "wkv_paged_prefill.cuh", "wkv_paged_f32.cuh",
                         "wkv_tcgen05.cuh"],
    "wkv_paged_rows.cu": [*PAGED, "wkv_paged_kv4.cuh", "wkv_paged_rows.cuh"],
    "wkv_paged_kv4.cu": [*PAGED, "wkv_paged_kv4.cuh", "wkv_paged_decode.cuh", "wkv_paged_decode_kv4.cuh"],
    "wkv_paged_pages.cu": [*PAGED, "wkv_paged_choose.cuh", "wkv_paged_decode.cuh"],
}
SOURCES = list(UNITS)
DEPS = sorted(set(SOURCES) | {d for deps in UNITS.values() for d in deps})
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]


def _mtime(path: str) -> float:
    return os.path.getmtime(path) if os.path.exists(path) else -1.0


def _stale() -> bool:
    return any(_mtime(os.path.join(CSRC, d)) > _mtime(LIB) for d in DEPS)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if force or _stale():
        nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
        extra = os.environ.get("WKV_NVCC_EXTRA", "").split()      # build-time tuning macros, e.g. -DWKV_RING_BYTES=49152
        os.makedirs(OBJ_DIR, exist_ok=True)

        def compile_unit(src: str) -> str:
            obj = os.path.join(OBJ_DIR, src[:-3] + ".o")
            newest = max(_mtime(os.path.join(CSRC, d)) for d in [src] + UNITS[src])
            if force or verbose or extra or _mtime(obj) < newest:
                cmd = [nvcc, *NVCC_FLAGS, *extra, *(["-Xptxas", "-v"] if verbose else []), "-c", "-o", obj + ".tmp", src]
                subprocess.run(cmd, check=True, cwd=CSRC)
                os.replace(obj + ".tmp", obj)
                if extra:                       # not an object that a later build without the macros may reuse
                    os.utime(obj, (0, 0))
            return obj

        with ThreadPoolExecutor(len(UNITS)) as pool:
            objs = list(pool.map(compile_unit, UNITS))
        subprocess.run([nvcc, *NVCC_FLAGS, "-shared", "-o", LIB + ".tmp", *objs], check=True, cwd=CSRC)
        os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
