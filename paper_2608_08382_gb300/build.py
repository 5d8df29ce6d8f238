"""Build the CUDA library in-tree: paper_2608_08382_gb300/_build/libllmvisor.so (sm_103a).

    python paper_2608_08382_gb300/build.py [--force]
"""

from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
OUT_DIR = os.path.join(HERE, "_build")
OUT = os.path.join(OUT_DIR, "libllmvisor.so")
SRCS = [os.path.join(HERE, "csrc", n) for n in ("lv_api.cu", "lv_kv.cu")]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _inputs():
    return (SRCS + glob.glob(os.path.join(HERE, "csrc", "*.cuh")) + glob.glob(os.path.join(HERE, "csrc", "*.h"))
            + [os.path.join(ROOT, "include", "llmvisor.h")])


def build(force: bool = False, extra=()) -> str:
    os.makedirs(OUT_DIR, exist_ok=True)
    if not force and os.path.exists(OUT):
        newest = max(os.path.getmtime(p) for p in _inputs())
        if os.path.getmtime(OUT) >= newest:
            return OUT
    tmp = OUT + f".tmp{os.getpid()}"
    objs = [f"{tmp}.{os.path.basename(src)}.o" for src in SRCS]
    # the translation units side by side
    jobs = [subprocess.Popen([nvcc(), *ARCH, "-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-c",
                              "-I", os.path.join(ROOT, "include"), "-o", obj, src, *extra])
            for src, obj in zip(SRCS, objs)]
    codes = [j.wait() for j in jobs]
    try:
        if any(codes):
            raise RuntimeError(f"nvcc failed: {dict(zip(SRCS, codes))}")
        subprocess.run([nvcc(), *ARCH, "-shared", "-o", tmp, *objs, "-lcudart"], check=True)
    finally:
        for obj in objs:
            if os.path.exists(obj):
                os.remove(obj)
    os.replace(tmp, OUT)
    return OUT


if __name__ == "__main__":
    print(build(force="--force" in sys.argv))
