"""GPU: a row whose map entry names no token is a row of zeros in the gated FFN's hidden values and in what comes from 4 bits also where its expert's weights
hold a NaN or an infinity, whichever kernel the number of rows selects."""
import numpy as np
import pytest
import torch

from paper_2407_00599_amd import api
from test_gpu_mx4 import store
from test_gpu_ragged_zero_rows import holes
from util import DEV

pytestmark = pytest.mark.gpu
BAD = [float("inf"), float("nan")]


def spoiled(W, bad):
    """one weight of every expert: its rows, those without a token apart, are not finite"""
    W[:, 3, 5] = bad
    return W


def check(hole, n, zero, lost):
    rows = torch.from_numpy(hole[:n])
    for t in zero:
        assert (t[:n][rows] == 0).all()
    for t in lost:
        assert not torch.isfinite(t[:n][~rows].float()).all(1).any()


# few rows in serving, small tiles, 192 x 256, 256 x 256; fp32
@pytest.mark.parametrize("dtype,ns,behind,M,H", [
    ("f32", (20, 0, 45, 9), 6, 136, 272), ("f32", (1,), 0, 64, 64), ("bf16", (20, 0, 45, 9), 6, 136, 272), ("bf16", (5, 9, 0, 1), 3, 520, 4400),
    ("bf16", (20, 9), 1, 520, 16400), ("bf16", (1010, 3, 12), 5, 72, 4104), ("bf16", (700, 0, 830), 20, 72, 4104)])
@pytest.mark.parametrize("bad", BAD)
def test_glu(dtype, ns, behind, M, H, bad):
    c, hole = holes(ns, behind, M, H, dtype, bad)
    n = c.offsets[-1]
    W1 = spoiled(c.stored(c.rng.standard_normal((c.E, M, 2 * H)) / np.sqrt(M)), bad)
    W2 = c.stored(c.rng.standard_normal((c.E, H, M)) / np.sqrt(H))
    A, Aserve, Y, Yserve, Z = c.fresh(c.R, H), c.fresh(c.R, H), c.fresh(c.R, M), c.fresh(c.R, M), c.fresh(c.R, 2 * H)
    ws = torch.empty(api.moe_ragged_glu_workspace_bytes(api.dtype_code(c.x), c.R, c.E, M, H, 1, 0) + 16, dtype=torch.uint8, device=DEV)
    shape = (c.off, c.R, c.E, M, H, 0, 1, api.MOE_ACT_SILU)
    api.moe_ragged_glu_fwd(*c.source(), W1, W2, *shape, None, Aserve, Yserve, ws)
    api.moe_ragged_glu_fwd(*c.source(), W1, W2, *shape, Z, A, Y, ws)
    check(hole, n, (A, Aserve, Z, Y, Yserve), (Z,))


# few rows (one and two groups of 16), tiles of 128 and of 256
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ns,behind,K,N", [((5, 9, 0, 1), 3, 520, 136), ((20, 9), 3, 520, 136), ((200, 0, 145, 9), 6, 136, 272), ((1300, 257), 4, 72, 8200)])
@pytest.mark.parametrize("bad", BAD)
def test_products_from_four_bits(ns, behind, K, N, dtype, bad):
    c, hole = holes(ns, behind, K, N, dtype, bad)
    W = spoiled(c.stored(c.rng.standard_normal((c.E, K, N)) / np.sqrt(K)), bad)
    xq, xs = store(c.x.view(1, *c.x.shape), False)
    Wq, Ws = store(W, True)
    Y = c.fresh(c.R, N)
    api.moe_ragged_gemm_mx4(xq, xs, c.S, c.inv, c.k, Wq, Ws, c.off, c.R, c.E, K, N, Y)
    check(hole, c.offsets[-1], (Y,), (Y,))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ns,behind,M,H", [((5, 9, 0, 1), 3, 520, 136), ((20, 9), 3, 520, 136), ((200, 0, 145, 9), 6, 136, 272), ((1300, 257), 4, 72, 4104)])
@pytest.mark.parametrize("bad", BAD)
def test_glu_from_four_bits(ns, behind, M, H, dtype, bad):
    c, hole = holes(ns, behind, M, H, dtype, bad)
    W1 = spoiled(c.stored(c.rng.standard_normal((c.E, M, 2 * H)) / np.sqrt(M)), bad)
    W2 = c.stored(c.rng.standard_normal((c.E, H, M)) / np.sqrt(H))
    (W1q, W1s), (W2q, W2s) = store(W1, True), store(W2, True)
    Y = c.fresh(c.R, M)
    ws = torch.empty(api.moe_ragged_glu_mx4_workspace_bytes(c.S, c.R, c.E, M, H), dtype=torch.uint8, device=DEV)
    api.moe_ragged_glu_mx4(c.x, c.S, c.inv, c.k, W1q, W1s, W2q, W2s, c.off, c.R, c.E, M, H, api.MOE_ACT_SILU, Y, ws)
    check(hole, c.offsets[-1], (Y,), (Y,))
