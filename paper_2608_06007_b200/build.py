"""Builds libtensorcast_b200.so (the C-ABI library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libtensorcast_b200.so")
SOURCES = ["exec.cu", "launch.cu", "staging.cu", "noalloc.cu", "plan_build.cpp", "ops_check.cpp", "kv_append.cu", "kv_gather.cu", "attn_decode.cu", "attn_prefix.cu", "attn_window.cu", "attn_singles.cu", "attn_chunk.cu", "attn_chunk_codes.cu", "attn_chunk_wide.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC,-Wall,-Wextra,-fvisibility=hidden"]


def _inputs():
    files = [os.path.join(INCLUDE, "tensorcast.h")]
    files += [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    return files


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > t for f in _inputs())


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile the library if it is missing or older than its sources; return its path."""
    if not force and not stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + f".{os.getpid()}.tmp"

    def run(cmd):
        if verbose:
            print(" ".join(cmd), file=sys.stderr)
        subprocess.check_call(cmd)

    with tempfile.TemporaryDirectory() as objects:
        made = [os.path.join(objects, s + ".o") for s in SOURCES]
        compile_ = [nvcc, *(["-Xptxas=-v"] if verbose else []), *NVCC_FLAGS, "-I", INCLUDE, "-I", CSRC, "-c"]
        with ThreadPoolExecutor(os.cpu_count() or 1) as workers:
            list(workers.map(lambda s, o: run([*compile_, "-o", o, os.path.join(CSRC, s)]), SOURCES, made))
        run([nvcc, *NVCC_FLAGS, "-shared", "-cudart", "static", "-o", tmp, *made])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
