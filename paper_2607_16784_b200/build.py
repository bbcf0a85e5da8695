"""Builds libroomie.so (sm_100a) in-tree with nvcc.  No JIT cache, no torch extension:
the shared library exports a plain C ABI (include/roomie.h) and is loaded with ctypes."""
from __future__ import annotations

import os
import subprocess

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libroomie.so")
SOURCES = ["roomie_api.cu", "roomie_library.cu", "roomie_pairs.cu", "roomie_place.cu", "roomie_optimal.cu",
           "roomie_serving.cu", "roomie_kv_append.cu", "roomie_kv_attention.cu", "roomie_kv_prompt.cu",
           "roomie_kv_pages.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "--fmad=true", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "roomie.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objs, running = [], []
    for src in SOURCES:                                   # one compiler per source, side by side
        obj = os.path.join(CSRC, src.replace(".cu", ".o"))
        cmd = [nvcc, *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        running.append((cmd, subprocess.Popen(cmd)))
        objs.append(obj)
    failed = [(p.returncode, cmd) for cmd, p in running if p.wait() != 0]
    if failed:
        raise subprocess.CalledProcessError(*failed[0])
    tmp = LIB + ".tmp%d" % os.getpid()
    subprocess.check_call([nvcc, "-shared", "-o", tmp, *objs, "-lcudart"])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
