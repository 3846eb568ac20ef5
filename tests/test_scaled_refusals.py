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


# ---------------------------------------------------------------- the binding, on CPU tensors, with nothing called behind it
@pytest.fixture
def calls(monkeypatch):
    """What the binding passes on to the library, by name; the tensors' device is taken for the current one."""
    made = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: made.append((name, a)) or 0

    monkeypatch.setattr(M, "load", Library)
    monkeypatch.setattr(M, "_on_device", lambda t, name: t.get_device())
    monkeypatch.setattr(M, "_stream_of", lambda stream, device: None)
    monkeypatch.setattr(M, "_stream", lambda stream: None)
    return made


def e4m3(rows, cols):
    return torch.zeros((1, 1), dtype=torch.uint8).view(torch.float8_e4m3fn).expand(rows, cols) if rows > 1000 or cols > 1000 else M.alloc_codes(rows, cols, device="cpu")[0]


def layer(K, N):
    h = C.c_void_p(0)
    h.K, h.N = K, N
    return h


@pytest.mark.parametrize("rows", [2**31, 2**32 + 3, 2**33])
def test_more_rows_than_the_library_counts_are_refused(calls, rows):
    """What passes 32 bits would arrive as another number of rows."""
    x, scales = torch.zeros((1, 8)).expand(rows, 8), torch.zeros((1, 1)).expand(1, rows)
    norm = M.make_residual_norm(8)
    for call in (lambda: M.mixaq_scaled_quantize(x, e4m3(rows, 8), scales), lambda: M.mixaq_scaled_linear_forward(layer(8, 8), x, x),
                 lambda: M.mixaq_residual_norm(norm, x, out=x), lambda: M.mixaq_scaled_linear_workspace_bytes(layer(8, 8), rows, torch.float32, torch.float32)):
        with pytest.raises(ValueError, match="2\\^30 rows"):
            call()
    assert not calls


def test_wider_matrices_than_the_library_counts_are_refused(calls):
    cols = 2**32 + 8                                      # (no such matrix is allocated: its values would be one, 0 apart)
    wide = torch.zeros((1, 1)).expand(1, cols)
    with pytest.raises(ValueError):
        M.mixaq_scaled_quantize(wide, e4m3(1, cols), torch.zeros((1, 1)).expand(cols // 128 + 1, 1))
    with pytest.raises(ValueError, match="channels"):
        M.make_residual_norm(cols)
    assert not calls


def test_a_gate_for_more_rows_than_there_can_be_is_a_gate_for_all(calls):
    x = torch.zeros((5, 8))
    for span in (2**31 - 1, 2**31, 2**32, 2**32 + 3, 2**63):
        norm = M.make_residual_norm(8, gate=torch.ones(1, 8), rows_per_gate=span)
        assert norm.desc.rows_per_gate == 2**31 - 1
        M.mixaq_residual_norm(norm, x, x, out=x)
    with pytest.raises(ValueError, match="rows_per_gate"):
        M.make_residual_norm(8, gate=torch.ones(1, 8), rows_per_gate=-1)


def test_a_norm_takes_rows_on_the_device_of_its_vectors(calls, monkeypatch):
    """Its vectors were on the current device when it was made; another one may be current when it is called."""
    with_gate, bare = M.make_residual_norm(8, gate=torch.ones(8)), M.make_residual_norm(8)
    gamma = M.make_residual_norm(8, pre_gamma=torch.ones(8))
    beta = M.make_residual_norm(8, post="layer", post_beta=torch.ones(8))
    monkeypatch.setattr(M, "_on_device", lambda t, name: 1)
    monkeypatch.setattr(M, "_rows", lambda *a: None)      # (x, y on device 1)
    x = torch.zeros((5, 8))
    for norm in (with_gate, gamma, beta):
        with pytest.raises(ValueError, match="vectors"):
            M.mixaq_residual_norm(norm, x, x, out=x)
    assert not calls
    M.mixaq_residual_norm(bare, x, x, out=x)              # without vectors it belongs to no device
    assert len(calls) == 1


def test_a_stream_of_another_device_is_refused(monkeypatch):
    class Stream:
        device_index, cuda_stream = 1, 0x1234

    assert M._stream_of(Stream, 1).value == 0x1234
    with pytest.raises(ValueError, match="stream"):
        M._stream_of(Stream, 0)


def test_a_workspace_has_the_bytes_it_says(calls):
    """An expanded tensor counts values that it has no memory for, a transposed or sliced one memory that belongs to others."""
    x = torch.zeros((5, 8))
    byte = torch.zeros(1, dtype=torch.uint8)
    for ws in (byte.expand(1 << 20), torch.zeros((64, 64)).t(), torch.zeros(64)[::2], torch.zeros((8, 8))[:, :4]):
        with pytest.raises(ValueError, match="workspace must be contiguous"):
            M.mixaq_scaled_linear_forward(layer(8, 8), x, torch.zeros((5, 8)), workspace=ws)
    assert not calls
    M.mixaq_scaled_linear_forward(layer(8, 8), x, torch.zeros((5, 8)), workspace=torch.zeros((8, 8))[2:])
    assert calls[0][1][5] == 6 * 8 * 4


def test_codes_have_room_for_whole_16_bytes(calls):
    """A layer reads a row's codes 16 at a time, those of the last row (or the only one, whose stride means nothing) too."""
    y = torch.zeros((1, 8))
    byte = lambda n: torch.zeros(n, dtype=torch.uint8).view(torch.float8_e4m3fn)
    scales = torch.ones((1, 3))
    for x in (byte(100).view(1, 100), byte(111).view(1, 111)[:, :100], byte(2 * 112 + 100).as_strided((3, 100), (112, 1)), byte(116)[16:].view(1, 100)):
        with pytest.raises(ValueError, match="room"):
            M.mixaq_scaled_linear_forward(layer(100, 8), x, y.expand(len(x), 8).contiguous(), x_scales=scales[:, :len(x)])
    assert not calls
    for x in (byte(112).view(1, 112)[:, :100], byte(3 * 112).as_strided((3, 100), (112, 1)), byte(128)[16:].view(1, 112)[:, :100], byte(100)[:0].view(0, 100)):
        M.mixaq_scaled_linear_forward(layer(100, 8), x, y.expand(len(x), 8).contiguous(), x_scales=scales[:, :len(x)])
    M.mixaq_scaled_linear_forward(layer(96, 8), byte(96).view(1, 96), y, x_scales=scales[:, :1])
    assert len(calls) == 5
    M.mixaq_scaled_quantize(torch.zeros((1, 100)), byte(100).view(1, 100), scales[:, :1])      # written without what is behind the columns


# ---------------------------------------------------------------- the library
def rows(data, stride=256, kind=2, scales=None, scale_stride=0):
    return M.Rows(data, stride, kind, scales, scale_stride)


VECTORS = ("post_gamma", "post_beta", "pre_gamma", "pre_beta", "gate")


@pytest.mark.parametrize("vector", VECTORS)
@pytest.mark.parametrize("written", ["y", "out", "scales"])
def test_norms_refuse_outputs_over_their_vectors(vector, written):
    """A vector that a row's results replace would be another one for the next row."""
    n, channels = 10, 200
    desc = M.ResidualNormDesc(channels, 1, 2, 3, 1e-5, 1e-5, 1.0)
    x, f, y, out, scales = (AT + (i << 20) for i in range(5))
    at = {"y": y, "out": out, "scales": scales}[written]
    size = {"y": (n - 1) * 512 + 400, "out": (n - 1) * 256 + 200, "scales": 4 * (16 + n)}[written]       # bytes from the first to the last
    length = 4 * channels * (4 if vector == "gate" else 1)                                              # gates: ceil(10 / 3)

    def call(where):
        p = M.ResidualNormParams(**{vector: where})
        return M.load().mixaq_residual_norm(C.byref(desc), C.byref(p), rows(x), rows(f), rows(y), rows(out, 256, 3, scales, 16), n, None)

    for where in (at, at + size - 4, at - length + 4):
        refused("%s and %s overlap" % ("y" if written == "y" else "out", vector), call(where))
