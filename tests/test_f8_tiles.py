"""Which tiles 8-bit floating point products run on: those that the GPU tests of the tiles are meant to run (CPU)."""
import ctypes

import pytest

from f8_tile_cases import HUGE
from paper_2607_05380_amd import tabpack


@pytest.mark.parametrize("case,layout", HUGE, ids=str)
def test_layout(case, layout):
    M, N, K, gate, fp32, pad, shift = case
    aligned = shift % 16 == 0 and (K + pad) % 16 == 0
    assert tabpack.debug_f8_matmul(M, N, K, gate, fp32, aligned) == layout


def test_refusals():
    out = [ctypes.byref(ctypes.c_int32()) for _ in range(3)]
    lib = tabpack.load_library()
    good = [16, 16, 128, -1, 0, 1]
    assert lib.pack_debug_f8_matmul(*good, *out) == 0
    for i, v in ((0, -1), (1, 0), (2, 0), (3, 3), (4, 2)):
        assert lib.pack_debug_f8_matmul(*(good[:i] + [v] + good[i + 1:]), *out) == -1
    assert lib.pack_debug_f8_matmul(*good, out[0], None, out[2]) == -1
