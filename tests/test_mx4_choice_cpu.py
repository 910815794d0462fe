"""Which kernel takes a product from 4 bits: the one for few rows (0) or tiles of 128 or 256."""
import ctypes

from paper_2407_00599_amd import api


def tile(R, E, N, K):
    f = api.lib()._ZN3moe8mx4_tileElili        # int moe::mx4_tile(int64_t R, int E, int64_t n, int K)
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_int64, ctypes.c_int, ctypes.c_int64, ctypes.c_int]
    return f(R, E, N, K)


def test_few_rows_are_bounded_whatever_the_number_of_experts():
    """That kernel reads an expert's weights again for every 16 rows of it, and all rows may be one expert's."""
    for E in (1, 2, 4, 8, 64, 256):
        for K, N in ((4096, 14336), (2048, 1024), (7168, 2048), (8, 8)):
            assert tile(1, E, N, K) == tile(32, E, N, K) == 0
            for R in (33, 64, 128, 1024, 4096):
                assert tile(R, E, N, K) in (128, 256), (R, E)
