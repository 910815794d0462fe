"""Sizes whose launch would have 2^32 threads or more are refused on the host, the ones next to them are not."""
import ctypes

import pytest

from paper_2407_00599_amd import api
from test_mx4_choice_cpu import tile

A = ctypes.c_void_p(0x1000)        # aligned dummy pointers: never dereferenced on these paths
U = ctypes.c_void_p(0x1004)        # misaligned: refused behind the sizes
EUNSUPPORTED, EALIGN = -2, -3


@pytest.mark.parametrize("dtype", [api.MOE_BF16, api.MOE_F32])
def test_store_and_load(dtype):
    L = api.lib()

    def both(G, rows, cols, tr):
        codes = {L.moe_mx4_store(U, dtype, G, rows, cols, tr, A, A, None), L.moe_mx4_load(U, A, G, rows, cols, tr, A, dtype, None)}
        assert len(codes) == 1
        return codes.pop()
    # pieces of 64 rows x 128 columns, 32 x 256, 16 x 512; transposed 512 rows x 128 columns
    for cols, rows, wide in ((8, 64, 1), (128, 64, 1), (136, 32, 1), (256, 32, 1), (264, 16, 1), (512, 16, 1), (520, 16, 2), (1032, 16, 3)):
        limit = rows * -(-(1 << 24) // wide)          # `wide` pieces beside each other
        for n, code in ((limit, EUNSUPPORTED), (limit - rows, EALIGN)):
            if n <= 1 << 31:
                assert both(1, n, cols, 0) == code, (cols, n)
    assert both(1 << 20, 1 << 31, 2147483640, 0) == EUNSUPPORTED           # 2^69 pieces
    assert both(1 << 4, 512, (1 << 27) + 128, 1) == EUNSUPPORTED and both(1 << 4, 512, (1 << 27) - 128, 1) == EALIGN


def test_products():
    L = api.lib()

    def gemm(R, E, K, N):
        return L.moe_ragged_gemm_mx4(U, A, 0, None, 1, A, A, A, R, E, K, N, A, api.MOE_BF16, None, 0, None)

    def glu(R, E, M, H):
        return L.moe_ragged_glu_mx4(U, api.MOE_BF16, 0, None, 1, A, A, A, A, A, R, E, M, H, 0, A, None, 0, None)
    # the kernel for few rows has a workgroup for every 64 columns of every expert, used or not; tiles only where there are rows
    assert tile(8, 8, 1 << 26, 8) == 0 and tile(8, 8, 1 << 27, 8) != 0
    assert gemm(8, 8, 8, 1 << 26) == EALIGN and gemm(8, 8, 8, 1 << 27) == EALIGN
    assert gemm(256, 256, 8, 1 << 22) == EALIGN and gemm(256, 256, 8, 1 << 24) == EUNSUPPORTED
    assert gemm(32, 32, 32, (1 << 27) - 8) == EUNSUPPORTED and glu(32, 32, 32, 1 << 26) == EUNSUPPORTED
    assert glu(32, 32, 32, 1 << 22) == EALIGN
