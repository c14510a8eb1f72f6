"""Builds libgsr.so (the C-ABI HIP library) in-tree with hipcc for gfx950, and the binding's helper that reads lists of torch tensors
(host code) with the host compiler."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libgsr.so")
MARSHAL = os.path.join(HERE, "libgsr_marshal.so")
SOURCES = ["gsr_graph.hip", "gsr_ops.hip", "gsr_layer.hip", "gsr_literal.hip", "gsr_optim.hip", "gsr_embed.hip",
           "gsr_lists.hip", "gsr_norm.hip", "gsr_classes.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",   # no packed-fp32 instructions
    # fuse a*b+c only where one source expression says so: the same helper inlined into two
    # kernels must round identically (records emitted by different kernels are bit-identical)
    "-ffp-contract=on",
    "-Wall", "-Wno-unused-variable", "-Wno-unused-but-set-variable",
    "-I", INCLUDE, "-I", CSRC,
]


def _hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def build_marshal(verbose: bool = True) -> str:
    """Compile gsr_marshal.cpp against the installed torch.  What an earlier build left goes first: it may fit another torch."""
    if os.path.exists(MARSHAL):
        os.remove(MARSHAL)
    import torch
    from torch.utils import cpp_extension
    includes = [*cpp_extension.include_paths(), sysconfig.get_paths()["include"]]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *(f"-I{i}" for i in includes),
           os.path.join(CSRC, "gsr_marshal.cpp"), "-o", MARSHAL, *(f"-L{i}" for i in cpp_extension.library_paths()),
           "-ltorch_python", "-ltorch_cpu", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    return MARSHAL


def build_library(verbose: bool = True) -> str:
    """Compile every HIP source for gfx950 and link libgsr.so, and build the binding's helper.  Always recompiles.  libgsr.so needs no torch: where
    the helper cannot be built (no torch, none of its headers, no host compiler) it is left out with a word on stderr, and the binding's
    calls on lists of tensors raise."""
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    hipcc = _hipcc()

    def compile_one(src: str) -> str:
        obj = os.path.join(objdir, src.replace(".hip", ".o"))
        cmd = [hipcc, *HIPCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        marshal = ex.submit(build_marshal, verbose)
        objs = list(ex.map(compile_one, SOURCES))
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    try:
        marshal.result()
    except (ImportError, OSError, subprocess.CalledProcessError) as e:
        print(f"{MARSHAL} was not built ({e}): calls on lists of tensors will raise", file=sys.stderr, flush=True)
    return LIB


if __name__ == "__main__":
    build_library()
    print(LIB)
