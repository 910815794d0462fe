"""GPU parity of the products from 4 bits and of the gated FFN served from them in the kernel for few rows: experts with more rows than go along with one
reading of the weights, many experts of which few have rows, all rows one expert's, the most rows that it takes and one more.  The tests, their oracle and
their bounds are those of test_gpu_mx4.py."""
import pytest

import test_gpu_mx4 as base
from test_mx4_choice_cpu import tile

pytestmark = pytest.mark.gpu

SIZES = [((20, 0, 1, 0, 2), 3, 520, 136, True), ((0, 32), 0, 264, 200, False), ((0,) * 65 + (3, 0, 27), 2, 136, 72, True), ((17, 1), 14, 1032, 328, True),
         ((0,) * 200 + (25,) + (0,) * 55, 7, 72, 264, True), ((31, 0, 0, 0, 1), 0, 2056, 64, False)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ns,behind,K,N,gather", SIZES)
def test_products(ns, behind, K, N, gather, dtype):
    assert tile(sum(ns) + behind, len(ns), N, K) == 0
    base.test_products(ns, behind, K, N, gather, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ns,behind,K,N,gather", [((20, 0, 1, 0, 2), 10, 520, 136, True), ((0,) * 65 + (3, 0, 27), 3, 136, 72, False)])
def test_products_of_one_row_more(ns, behind, K, N, gather, dtype):
    assert tile(sum(ns) + behind, len(ns), N, K) == 128
    base.test_products(ns, behind, K, N, gather, dtype)


@pytest.mark.parametrize("dtype,act", [("f32", "gelu"), ("bf16", "silu")])
@pytest.mark.parametrize("ns,behind,M,H,gather", SIZES)
def test_glu(ns, behind, M, H, gather, dtype, act):
    base.test_glu(ns, behind, M, H, gather, dtype, act)
