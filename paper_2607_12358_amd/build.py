"""Builds libacid.so (gfx950) in-tree with hipcc.

    python -m paper_2607_12358_amd.build        # or __graft_entry__.build()

Every HIP source is compiled for gfx950 with packed-fp32 instructions
disabled; the gate is host code compiled without floating-point contraction.
What the binding does natively is a Python module of its own, _binding.so.
Objects go to ``_build/``; the shared libraries land next to this file.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libacid.so")
BINDING = os.path.join(PKG, "_binding.so")
ARCH = "gfx950"

HIP_SOURCES = ["elementwise.hip", "temb.hip", "gemm.hip", "attention.hip", "runtime.hip",
               "noalloc.hip", "linear_attention.hip", "residual_norm.hip", "linear_w4.hip"]
HOST_SOURCES = ["gate.cpp"]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found")


def _flags_common():
    return ["-O3", "-fPIC", "-std=c++17", f"-I{INCLUDE}", f"-I{CSRC}"]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    path = os.path.join(CSRC, src)
    if src.endswith(".hip"):
        cmd = [hipcc(), *_flags_common(), f"--offload-arch={ARCH}", "-x", "hip",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-munsafe-fp-atomics", "-c", path, "-o", obj]
    else:
        cmd = [hipcc(), *_flags_common(), "-ffp-contract=off", "-fno-fast-math",
               "-c", path, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def _link(target: str, *args: str) -> None:
    tmp = target + ".tmp"
    cmd = [hipcc(), "-shared", "-fPIC", *args, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, target)


def build(verbose: bool = True) -> str:
    os.makedirs(BUILD, exist_ok=True)
    srcs = HIP_SOURCES + HOST_SOURCES
    with cf.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(_compile, srcs))
    _link(LIB, f"--offload-arch={ARCH}", *objs)
    _link(BINDING, *_flags_common(), f"-I{sysconfig.get_paths()['include']}",
          os.path.join(CSRC, "binding.cpp"))
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build()
    sys.exit(0)
