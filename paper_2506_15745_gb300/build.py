"""Builds libipv.so (the CUDA path) in-tree for sm_103a with nvcc.

The translation units compile in parallel; the CUDA runtime is linked
statically so the library has no dependency beyond the driver.
"""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libipv.so")
SOURCES = ["api.cu", "score.cu", "select.cu", "gather.cu", "pool.cu", "combine.cu", "append.cu", "window.cu", "noalloc.cu",
           "paged.cu", "paged_rows.cu", "attend_rows.cu", "attend_tiles.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]


def _stale(out: str, deps: list[str]) -> bool:
    return not os.path.exists(out) or any(os.path.getmtime(d) > os.path.getmtime(out) for d in deps)


def build(force: bool = False, extra_flags: list[str] | None = None, verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, "ipv_common.cuh"), os.path.join(CSRC, "pass_device.cuh"),
               os.path.join(CSRC, "paged.cuh"), os.path.join(CSRC, "attend_share.cuh"),
               os.path.join(INCLUDE, "ipv.h")]
    procs, objs = [], []
    for src in SOURCES:
        path = os.path.join(CSRC, src)
        obj = os.path.join(OBJ, src.replace(".cu", ".o"))
        objs.append(obj)
        if force or _stale(obj, [path] + headers):
            cmd = ["nvcc", *ARCH, *FLAGS, *(extra_flags or []), "-c", path, "-o", obj]
            if verbose:
                print(" ".join(cmd), file=sys.stderr)
            procs.append((src, subprocess.Popen(cmd)))
    failed = [src for src, p in procs if p.wait() != 0]
    if failed:
        raise RuntimeError(f"nvcc failed for {failed}")
    if force or procs or _stale(LIB, objs):
        subprocess.run(["nvcc", *ARCH, "-shared", "-o", LIB, *objs], check=True)
    return LIB


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose=True,
          extra_flags=["-Xptxas", "-v"] if "--ptxas-v" in sys.argv else None)
