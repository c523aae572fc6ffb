"""Builds libpdattn.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB_DIR = os.path.join(HERE, "lib")
LIB = os.path.join(LIB_DIR, "libpdattn.so")
SOURCES = ["pdattn_api.cu", "ops_api.cu", "prefill_api.cu", "scored_api.cu", "host_common.cu", "partition.cpp"]
HEADERS = ["kernels.cuh", "host_common.h", "common.cuh", "tile_bf16.cuh", "tile_fp8.cuh", "decode.cuh", "prefix_mma.cuh",
           "prefix_umma.cuh", "aux_kernels.cuh", "rope.cuh", "pages.cuh", "prefill_umma.cuh", "umma.cuh", "scored.h", "partition.h", os.path.join("..", "..", "include", "pdattn.h")]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def source_fingerprint() -> str:
    """sha256 over the kernel and host sources the library is built from (in a fixed order): names a build
    without needing the version control history, e.g. to tie a profile summary to the kernels it measured."""
    import hashlib
    h = hashlib.sha256()
    for f in sorted(SOURCES + HEADERS):
        path = os.path.join(CSRC, f)
        h.update(os.path.basename(f).encode())
        with open(path, "rb") as fh:
            h.update(fh.read())
    return h.hexdigest()


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps if os.path.exists(d))


def build(force: bool = False, verbose: bool = False, defines=(), out: str = None) -> str:
    """defines / out build a tuning variant (e.g. defines=["PDATTN_NCW=4"]) to another path."""
    target = out or LIB
    if out is None and not force and not needs_build():
        return LIB
    os.makedirs(os.path.dirname(target), exist_ok=True)
    tmp = target + ".tmp%d" % os.getpid()
    cmd = [_nvcc(), "-std=c++17", "-O3", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
           "-t", "0", "-Xcompiler", "-fPIC", "-shared", "-cudart", "static", "-o", tmp]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += ["-D" + d for d in defines]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    subprocess.check_call(cmd)
    os.replace(tmp, target)
    return target


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
