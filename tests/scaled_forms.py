"""The library's own rule of which kernel takes a linear layer in 8-bit float (csrc/scaled_forms.h), built for the host, and the sizes that the
GPU tests compare with the reference."""
import ctypes
import os
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_19131_amd", "csrc")
NAMES = ("few", "mid", "split", "tile", "large")

_SOURCE = r'''
#include "scaled_forms.h"
extern "C" int form(int M, int KB, int NB, int gelu, int exact, long long ldx) { return mixaq::scaled_form(M, KB, NB, gelu, exact, ldx); }
extern "C" int inside(int M, int KB, int NB) { return mixaq::quantized_inside(M, KB, NB); }
'''


def _build():
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "forms.cpp"), os.path.join(d, "forms.so")
        with open(src, "w") as f:
            f.write(_SOURCE)
        subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-fPIC", "-shared", "-I", CSRC, "-o", so, src], check=True)
        lib = ctypes.CDLL(so)
        lib.form.argtypes = [ctypes.c_int] * 5 + [ctypes.c_longlong]
        return lib


lib = _build()


def blocks(n):
    return -(-n // 128)


def form(rows, K, N, kind, gelu=False, ldx=None):
    """kind: of the results."""
    return NAMES[lib.form(rows, blocks(K), blocks(N), gelu, kind != "bf16", -(-K // 16) * 16 if ldx is None else ldx)]


def inside(rows, K, N):
    """Whether values are quantized on their way into the product."""
    return bool(lib.inside(rows, blocks(K), blocks(N)))


# rows, K, N: every kernel with K that ends inside 16 codes, between two 16s of a block, at a block; outputs that end inside a block and an odd number of
# blocks (of two that a large tile takes); more than 32 blocks of K
SIZES = [
    (1, 1000, 333), (16, 4400, 130), (40, 1024, 512), (130, 1000, 333),                                     # few
    (513, 1024, 1024), (700, 1500, 700), (300, 4000, 600), (256, 4400, 520),                                # mid
    (2000, 500, 600), (2000, 784, 600), (2010, 640, 512), (1300, 4500, 1200),                               # split
    (6000, 100, 512), (6200, 208, 640), (5000, 384, 700), (2600, 300, 1111),                                # tile
    (8200, 784, 1500), (8500, 790, 1400), (8192, 896, 1536), (12300, 400, 1130), (7000, 1000, 2000),        # large
]
KINDS = ("f32", "f16", "bf16", "e4m3")
