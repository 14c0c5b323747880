"""Builds the C-ABI shared library ``liblrgd.so`` in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblrgd.so")
SOURCES = ["lrgd_api.cu", "lrgd_gate_api.cu", "lrgd_class_api.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xptxas", "-v"]


def _newest_source_mtime() -> float:
    paths = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    paths.append(os.path.join(os.path.dirname(HERE), "include", "lrgd.h"))
    return max(os.path.getmtime(p) for p in paths)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile if the library is missing or older than any source.  Returns the library path."""
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source_mtime():
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    tmp = LIB + f".tmp{os.getpid()}"
    objects = [f"{tmp}.{i}.o" for i in range(len(SOURCES))]
    compiles = [[nvcc, *NVCC_FLAGS, "-c", "-o", obj, os.path.join(CSRC, src)] for obj, src in zip(objects, SOURCES)]
    try:
        # the sources are compiled side by side, then linked
        procs = [subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for cmd in compiles]
        outs = [p.communicate()[0] for p in procs]
        for cmd, proc, out in zip(compiles, procs, outs):
            if verbose or proc.returncode != 0:
                sys.stderr.write(out)
            if proc.returncode != 0:
                raise RuntimeError("nvcc failed: " + " ".join(cmd))
        link = [nvcc, *NVCC_FLAGS, "-shared", "-o", tmp, *objects]
        proc = subprocess.run(link, capture_output=True, text=True)
        if proc.returncode != 0:
            sys.stderr.write(proc.stdout + proc.stderr)
            raise RuntimeError("nvcc failed: " + " ".join(link))
    finally:
        for obj in objects:
            if os.path.exists(obj):
                os.remove(obj)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
