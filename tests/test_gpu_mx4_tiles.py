"""GPU parity of the products from 4 bits and of the gated FFN served from them in tiles of 256 x 256 (test_gpu_mx4.py has the kernel for few rows and
tiles of 128 x 128): each size is one for which the dispatch chooses them, with k tiles that are full, cut short and a single one.  The tests, their
oracle and their bounds are those of test_gpu_mx4.py."""
import pytest

import test_gpu_mx4 as base

pytestmark = pytest.mark.gpu


# rows per expert, rows behind, K, N, gather
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ns,behind,K,N,gather", [((1300, 257), 0, 72, 8200, True), ((700, 0, 900, 1), 5, 776, 7176, True), ((900, 600), 30, 1024, 8200, False)])
def test_products(ns, behind, K, N, gather, dtype):
    base.test_products(ns, behind, K, N, gather, dtype)


@pytest.mark.parametrize("dtype,act", [("f32", "gelu"), ("bf16", "silu"), ("bf16", "gelu")])
@pytest.mark.parametrize("ns,behind,M,H,gather", [((1300, 257), 3, 72, 4104, True), ((600, 0, 830), 0, 520, 2056, False)])
def test_glu(ns, behind, M, H, gather, dtype, act):
    base.test_glu(ns, behind, M, H, gather, dtype, act)
