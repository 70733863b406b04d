"""Which tiles 8-bit floating point products run on: those that the GPU tests of the tiles are meant to run (CPU)."""
import ctypes

import pytest

from f8_tile_cases import ALL
from paper_2607_05380_amd import tabpack


@pytest.mark.parametrize("case,layout", ALL, ids=str)
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


@pytest.mark.parametrize("M,N,K,gate", [(300, 8192, 20_000, None), (300, 8192, 20_000, "silu"), (1024, 4096, 16_384, "gelu"),
                                        (600, 2040, 40_016, None), (260, 520, 16_400, None), (3000, 1023, 1023, "silu"),
                                        (512, 2048, 65_536, "relu"), (8192, 8192, 8192, None)])
def test_workspace_serves_either_type(M, N, K, gate):
    """A workspace is asked for without the results' type: it holds the partial sums of both."""
    n = ctypes.c_size_t()
    code = -1 if gate is None else tabpack.ACTIVATIONS[gate]
    assert tabpack.load_library().pack_f8_matmul_workspace_size(M, N, K, code, ctypes.byref(n)) == 0
    for fp32 in (False, True):
        for aligned in (False, True):
            _, splits, _ = tabpack.debug_f8_matmul(M, N, K, gate, fp32, aligned)
            assert splits == 1 or n.value >= splits * M * N * (8 if gate else 4)
