"""The output tile and parts of K that a product of e4m3 operands takes, from the
library's own rule (csrc/fp8_form.h compiled for the host), so that a test can state which
kernel its sizes reach."""
import ctypes as C
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TILES = ("rows", "256x256", "128x128", "64x64")

SRC = """
#include "fp8_form.h"
extern "C" void form(int64_t M, int64_t N, int64_t K, int exact, int64_t cus, int64_t* out) {
  const acid::Fp8Form f = acid::fp8_form(M, N, K, exact != 0, cus);
  out[0] = (int)f.tile;
  out[1] = f.split;
  out[2] = f.floats;
}
"""


@functools.lru_cache(None)
def _lib():
    d = tempfile.mkdtemp()
    src, so = os.path.join(d, "form.cpp"), os.path.join(d, "form.so")
    with open(src, "w") as f:
        f.write(SRC)
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2607_12358_amd", "csrc"), src, "-o", so], check=True)
    return C.CDLL(so)


def fp8_form(M, N, K, exact=False, cus=256):
    """(tile, parts of K, floats of workspace)"""
    out = (C.c_int64 * 3)()
    _lib().form(C.c_int64(M), C.c_int64(N), C.c_int64(K), int(exact), C.c_int64(cus), out)
    return TILES[out[0]], int(out[1]), int(out[2])
