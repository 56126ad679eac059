"""Builds libtfno.so (the HIP library) in-tree with hipcc for gfx950, and _marshal.so (calls from Python) with the host's compiler.

Usage: ``python -m paper_2504_11681_amd.build``  (no GPU needed: hipcc cross-compiles).
"""
from __future__ import annotations

import concurrent.futures
import glob
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libtfno.so")
MARSHAL = os.path.join(HERE, "_marshal.so")

# packed FP32 instructions are switched off for all device code in this library
HIPCC_FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-fno-gpu-rdc",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-Wno-unused-command-line-argument", "-Wno-unknown-warning-option"]


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, os.path.basename(src) + ".o")
    cmd = ["hipcc", *HIPCC_FLAGS, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def _run(cmd, what: str) -> None:
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{r.stdout}\n{r.stderr}")


def _build_marshal() -> bool:
    """_marshal.so, which the operators along time are called through from Python; without torch there is nothing to build it for."""
    try:
        import torch
    except ImportError:
        return False
    root = os.path.dirname(torch.__file__)
    include, lib = os.path.join(root, "include"), os.path.join(root, "lib")
    _run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
          "-isystem", include, "-isystem", os.path.join(include, "torch", "csrc", "api", "include"), "-isystem", sysconfig.get_paths()["include"],
          os.path.join(CSRC, "marshal.cpp"), "-o", MARSHAL, f"-L{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-ldl"], "marshal.cpp")
    return True


def build(verbose: bool = True, jobs: int = 8) -> str:
    """The library first: it needs hipcc alone, and is there whatever becomes of _marshal.so."""
    os.makedirs(OBJ, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")))
    with concurrent.futures.ThreadPoolExecutor(max_workers=jobs) as ex:
        marshal = ex.submit(_build_marshal)
        objs = list(ex.map(_compile, srcs))
        _run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB], "link")
    both = marshal.result()
    if verbose:
        print(f"built {LIB} from {len(srcs)} sources, and {MARSHAL if both else 'no _marshal.so, since there is no torch'}", file=sys.stderr)
    return LIB


if __name__ == "__main__":
    build()
