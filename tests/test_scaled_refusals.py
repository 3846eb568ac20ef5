"""Calls of the 8-bit float layers and norms at the ends of what their arguments can say: refused before any GPU call.  CPU only."""
import ctypes as C
import os
import subprocess
import sys

import pytest
import torch

from paper_2507_19131_amd import binding as M

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHAPE = -2
AT, FAR = 1 << 20, 1 << 56                                # addresses that no call may touch


def refused(words, rc):
    assert rc == SHAPE and words in M.load().mixaq_last_error().decode(), (rc, M.load().mixaq_last_error())


@pytest.mark.parametrize("columns", [2**31 - 1, 2**31 - 127, 2**31 - 128])
def test_rows_of_nearly_2_31_columns_are_counted_in_blocks(columns):
    """Too many blocks for one call, whichever way they are counted; in a process of its own, since a wrong count made the host search for ever."""
    code = """
import sys; sys.path.insert(0, %r)
from paper_2507_19131_amd import binding as M
n = 1 << 15
x, q = M.Rows(%d, 1 << 31, 2, None, 0), M.Rows(%d, 1 << 31, 3, %d, n)
rc = M.load().mixaq_scaled_quantize(x, n, %d, 1, q, None)
assert rc == -2 and b"too many" in M.load().mixaq_last_error(), (rc, M.load().mixaq_last_error())
""" % (ROOT, AT, FAR, FAR << 1, columns)
    subprocess.run([sys.executable, "-c", code], check=True, timeout=120)
