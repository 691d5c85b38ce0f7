"""Build libsignsgd.so (the C-ABI CUDA library) for sm_100a with nvcc, in tree.

    python -m paper_1810_05291_b200.build [--force] [--verbose]

nvcc cross-compiles without a GPU. Objects go to ``_build/`` at the repository root; the
shared library is written next to this file so that it travels with the source tree.
"""

from __future__ import annotations

import argparse
import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsignsgd.so")
OBJ_DIR = os.path.join(ROOT, "_build", "signsgd")

SOURCES = ["abi.cu", "step_f32.cu", "step_bf16.cu", "vote_apply.cu", "noalloc.cu", "ternary.cu", "exchange_flags.cu",
           "act8.cu", "weight_grad8.cu", "losses.cu"]
HEADERS = ["bitslice.cuh", "common.cuh", "step_kernel.cuh", "step_oct_kernel.cuh", "exchange.cuh", "train.cuh", "act8.cuh", "tcgen05.cuh",
           os.path.join("..", "..", "include", "signsgd.h"), os.path.join("..", "..", "include", "signsgd_train.h")]

# -fmad=false: no multiply-add contraction anywhere (the arithmetic also uses explicitly
# rounded intrinsics); no -use_fast_math, denormals kept. The training operators are compared with
# a tolerance, not bit for bit, and may contract.
NVCC_FLAGS = ["-std=c++17", "-O3", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden"]
CONTRACTED = ("act8.cu", "weight_grad8.cu", "losses.cu")


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found; cannot build libsignsgd.so")
    return exe


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    os.makedirs(OBJ_DIR, exist_ok=True)
    nvcc = _nvcc()
    extra = ["-Xptxas", "-v"] if verbose else []

    def compile_one(src: str) -> str:
        obj = os.path.join(OBJ_DIR, os.path.splitext(src)[0] + ".o")
        contract = [] if src in CONTRACTED else ["-fmad=false"]
        cmd = [nvcc] + NVCC_FLAGS + contract + extra + ["-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if verbose or r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed on %s" % src)
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB + ".tmp.%d" % os.getpid()
    cmd = [nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("link failed")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--force", action="store_true")
    ap.add_argument("--verbose", action="store_true")
    a = ap.parse_args()
    print(build(force=a.force, verbose=a.verbose))
