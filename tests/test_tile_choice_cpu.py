"""The sizes of the tests of large tiles are sizes for which the dispatch chooses those tiles: the rules that the launches ask, asked here."""
import ctypes

import pytest

import test_gpu_glu
from paper_2407_00599_amd import api
from test_mx4_choice_cpu import tile as tile4


class Tile(ctypes.Structure):
    _fields_ = [("m", ctypes.c_int), ("n", ctypes.c_int)]


def tile(R, E, K, N, wide=False):
    f = api.lib()._ZN3moe9rows_tileEiiiib        # moe::TilePlan moe::rows_tile(int R, int E, int K, int N, bool wide)
    f.restype, f.argtypes = Tile, [ctypes.c_int] * 4 + [ctypes.c_bool]
    t = f(R, E, K, N, wide)
    return t.m, t.n


T256, T192, T128, T64x128, T64 = (256, 256), (192, 256), (128, 128), (64, 128), (64, 64)
# first product, gradients of g and u; or dX in the merged backward launch
FIRST = [(T256, T128), (T192, T128), (T256, T256), (T192, T192), (T64x128, T64), (T64x128, T64x128)]
MERGED = [T256, T256, T256, T128]


@pytest.mark.parametrize("size,want", list(zip(test_gpu_glu.LARGE, FIRST + MERGED)), ids=str)
def test_gated(size, want):
    ns, behind, M, H, n_esp = size[:5]
    R, E, Hl = sum(ns) + behind, len(ns), H // n_esp
    if isinstance(want[0], tuple):
        assert (tile(R, E, M, 2 * Hl), tile(R, E, M, Hl)) == want
    else:
        got = tile(R, E, 2 * Hl, M, True)
        assert got == want or {got, want} == {T256, T192}         # the launch takes 256 rows for either


def test_the_sizes_are_all_there():
    assert len(test_gpu_glu.LARGE) == len(FIRST) + len(MERGED)


# rows, experts, summed, columns: those of test_gpu_mx4_tiles.py, of the gated FFN its first product; but the last one of it, 1430 rows x 520 x 2 * 2056,
# runs in tiles of 128 (test_gpu_mx4_tiles_glu.py has such a call in tiles of 256)
@pytest.mark.parametrize("R,E,K,N", [(1557, 2, 72, 8200), (1606, 4, 776, 7176), (1530, 2, 1024, 8200), (1560, 2, 72, 2 * 4104)])
def test_from_four_bits(R, E, K, N):
    assert tile4(R, E, N, K) == 256


# those of test_gpu_mx4.py that have more than 32 rows
@pytest.mark.parametrize("R,E,K,N", [(91, 5, 264, 136), (225, 5, 128, 256), (325, 3, 520, 328), (153, 100, 64, 72), (814, 2, 1032, 72), (810, 3, 520, 520),
                                     (1557, 2, 264, 776), (260, 3, 264, 2 * 520), (833, 3, 128, 400), (1430, 3, 520, 2 * 2056)])
def test_from_four_bits_in_small_tiles(R, E, K, N):
    assert tile4(R, E, N, K) == 128
