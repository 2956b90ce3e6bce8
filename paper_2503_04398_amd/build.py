"""Build libsemmoe.so (HIP kernels + C ABI) for gfx950, in-tree.

    python -m paper_2503_04398_amd.build

hipcc cross-compiles without a GPU.  Objects go to paper_2503_04398_amd/_build/, the library to
paper_2503_04398_amd/lib/libsemmoe.so.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIBDIR = os.path.join(HERE, "lib")
LIB = os.path.join(LIBDIR, "libsemmoe.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

SOURCES = ["common.hip", "gemm.hip", "route.hip", "hist.hip", "reshuffle.hip", "dispatch.hip", "ffn.hip",
           "combine.hip", "rows_grad.hip", "gemm_nn.hip", "adapters.hip", "gemm_i8.hip", "ffn_i8.hip", "rows_i8.hip", "norm.hip", "request.hip", "probe.hip",
           "place.cpp"]

HIP_FLAGS = ["-O3", "--offload-arch=gfx950", "-fPIC", "-std=c++17", "-Wall", "-Wno-unused-function", "-Wno-inline-asm",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",   # no packed-fp32 instructions
             "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]
CXX_FLAGS = ["-O2", "-fPIC", "-std=c++17", "-Wall", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def _run(cmd):
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in p.stdout.splitlines() if "packed-fp32-ops" not in l)
    if p.returncode != 0:
        raise RuntimeError("command failed: %s\n%s" % (" ".join(cmd), out))
    return out


def _compile(src):
    obj = os.path.join(BUILD, src.rsplit(".", 1)[0] + ".o")
    path = os.path.join(CSRC, src)
    if src.endswith(".hip"):
        out = _run([HIPCC] + HIP_FLAGS + ["-c", path, "-o", obj])
    else:
        out = _run(["g++"] + CXX_FLAGS + ["-c", path, "-o", obj])
    return obj, out


def build(verbose: bool = True) -> str:
    os.makedirs(BUILD, exist_ok=True)
    os.makedirs(LIBDIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        results = list(ex.map(_compile, SOURCES))
    for obj, out in results:
        if verbose and out.strip():
            print(out)
    objs = [o for o, _ in results]
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs)
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build()
    sys.exit(0)
