"""The library's own rule of which kernel takes a linear layer on int8 codes (csrc/token_forms.h), built for the host, and the sizes that the GPU tests compare with
the reference."""
import ctypes
import os
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_19131_amd", "csrc")
NAMES = ("few", "mid", "split", "tile", "wide")

_SOURCE = r'''
#include "token_forms.h"
extern "C" int form(int M, int KB, int NB, int experts, int sorted, long long reach) { return mixaq::token_form(M, KB, NB, experts, sorted, reach); }
extern "C" int inside(int M, int K, int NB, int experts, int sorted) { return mixaq::token_quantized_inside(M, K, NB, experts, sorted); }
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


def form(rows, K, N, experts=0, stride=None):
    """experts: of rows sorted by expert."""
    stride = -(-K // 16) * 16 if stride is None else stride
    return NAMES[lib.form(rows, blocks(K), blocks(N), max(experts, 1), experts > 0, stride * (rows if experts else 128))]


def inside(rows, K, N, experts=0):
    """Whether values are quantized on their way into the product."""
    return bool(lib.inside(rows, K, blocks(N), max(experts, 1), experts > 0))


# rows, K, N: K that ends inside 16 codes, a step of 32, a stage of 64 and a block; outputs that end inside 16, 64 and 128, an odd number of blocks
SIZES = [
    (1, 1, 1), (1, 1000, 333), (3, 16, 8), (15, 4400, 130), (16, 128, 16), (17, 127, 129), (40, 1024, 512), (130, 1000, 333), (16, 40, 20000), (1024, 700, 300),        # few
    (300, 100, 600), (700, 1500, 200), (513, 784, 1030),                                                                                                             # mid, but the last
    (1100, 640, 1024), (1000, 90, 1300),                                                                                                                              # split
    (2100, 384, 1500), (4800, 96, 400), (13000, 1050, 100), (4200, 65, 700),                                                                                          # tile
    (9000, 790, 1300), (13000, 129, 700), (8500, 400, 1024),                                                                                                          # wide
]
# experts, rows, K, N, experts without rows
SORTED = [
    (1, 1, 64, 40, ()), (4, 3, 300, 200, ()), (8, 16, 1000, 333, (0,)), (33, 64, 128, 130, (3, 32)), (300, 2000, 40, 33, (150,)), (40, 500, 300, 260, (7,)),            # few
    (1, 700, 200, 300, ()), (8, 900, 384, 500, (0, 3, 7)), (5, 2500, 257, 130, (4,)), (64, 6000, 130, 70, (10, 11, 12)), (70, 5000, 96, 64, (0, 63, 64, 69)),           # tile
    (3, 9000, 500, 700, ()), (16, 9000, 300, 1030, (3, 15)), (130, 9000, 200, 140, (0, 64, 129)), (70, 9000, 160, 270, ()),                                           # tile, wide
]
