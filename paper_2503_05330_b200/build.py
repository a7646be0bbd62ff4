"""Builds ``libsdms.so`` (the CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsdms.so")
OBJECTS = os.path.join(HERE, "_build")
SOURCES = ["api.cu", "append.cu", "match.cu", "dag.cu", "dag_wide.cu", "beams.cu", "fuzzy.cu", "match_static.cu",
           "decode_api.cu", "kv.cu", "beam_select.cu", "attend.cu"]
HEADERS = ["sdms_dev.cuh", "sdms_internal.h", "append_dev.cuh", "wide_dev.cuh", "beam_dev.cuh", "beam_plan.h", "decode_internal.h", "decode_dev.cuh", "attend_plan.h"]


def _newest(files) -> float:
    return max(os.path.getmtime(f) for f in files)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles what is older than its source (or, with force, everything), a process per file, and links it."""
    headers = [os.path.join(CSRC, f) for f in HEADERS] + [os.path.join(ROOT, "include", "sdms.h")]
    sources = [os.path.join(CSRC, f) for f in SOURCES]
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest(sources + headers):
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC",
             "-I", os.path.join(ROOT, "include"), "-I", CSRC] + (["-Xptxas", "-v"] if verbose else [])
    os.makedirs(OBJECTS, exist_ok=True)

    def compile_one(source):
        obj = os.path.join(OBJECTS, os.path.basename(source) + ".o")
        if force or not os.path.exists(obj) or os.path.getmtime(obj) < _newest([source] + headers):
            part = f"{obj}.{os.getpid()}"
            subprocess.check_call([nvcc, *flags, "-c", source, "-o", part])
            os.replace(part, obj)
        return obj

    with ThreadPoolExecutor(max(1, min(len(sources), os.cpu_count() or 1))) as pool:
        objects = list(pool.map(compile_one, sources))
    part = f"{LIB}.{os.getpid()}"
    subprocess.check_call([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", *objects, "-o", part])
    os.replace(part, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
