"""GPU: rows among an expert's own whose map entry names no token (negative, or past the last one) are rows of zeros in the gated FFN and in the calls
from 4 bits too, also where token 0, which stands in for them, is not finite."""
import numpy as np
import pytest
import torch

import four_bits
import test_gpu_ragged as base
from oracle import ragged_oracle as O
from paper_2407_00599_amd import api
from test_gpu_mx4 import store
from test_gpu_ragged_zero_rows import holes
from util import DEV

pytestmark = pytest.mark.gpu
BAD = [float("inf"), float("nan")]


# small tiles, few rows in serving, 192 x 256, 256 x 256
@pytest.mark.parametrize("dtype,ns,behind,M,H", [
    ("f32", (20, 0, 45, 9), 6, 136, 272), ("bf16", (20, 0, 45, 9), 6, 136, 272), ("bf16", (5, 9, 0, 1), 3, 520, 4400),
    ("bf16", (1010, 3, 12), 5, 72, 4104), ("bf16", (700, 0, 830), 20, 72, 4104)])
@pytest.mark.parametrize("bad", BAD)
def test_glu(dtype, ns, behind, M, H, bad):
    c, hole = holes(ns, behind, M, H, dtype, bad)
    E, R, off = c.E, c.R, c.offsets
    n = off[-1]
    W1 = c.stored(c.rng.standard_normal((E, M, 2 * H)) / np.sqrt(M))
    W2 = c.stored(c.rng.standard_normal((E, H, M)) / np.sqrt(H))
    dY = c.stored(c.rng.standard_normal((R, M)))
    A, Y, Yserve, dX, Z = c.fresh(R, H), c.fresh(R, M), c.fresh(R, M), c.fresh(R, M), c.fresh(R, 2 * H)
    dW1, dW2 = c.fresh(E, M, 2 * H), c.fresh(E, H, M)
    ws = torch.empty(max(api.moe_ragged_glu_workspace_bytes(api.dtype_code(c.x), R, E, M, H, 1, b) for b in (0, 1)) + 16, dtype=torch.uint8, device=DEV)
    shape = (c.off, R, E, M, H, 0, 1, api.MOE_ACT_SILU)
    api.moe_ragged_glu_fwd(*c.source(), W1, W2, *shape, None, c.fresh(R, H), Yserve, ws)
    api.moe_ragged_glu_fwd(*c.source(), W1, W2, *shape, Z, A, Y, ws)
    api.moe_ragged_glu_bwd(dY, *c.source(), Z, W1, W2, *shape, dX, dW1, dW2, ws)
    for t in (A, Y, Yserve, Z, dX):
        assert (t[:n][torch.from_numpy(hole[:n])] == 0).all()
    # the other rows and the gradients are those of a token matrix that holds zeros there: tolerance of the tensors as a whole, 2^-6 for six
    # roundings of 2^-8 in bf16 whose errors add up like their squares, a thousandth of that for fp32's 2^-24
    tol = 2.0 ** -6 if dtype == "bf16" else 2.0 ** -16
    w1, w2, g, z = base.host(W1), base.host(W2), base.host(dY), base.host(Z)
    g[n:] = z[n:] = 0
    y = O.glu_fwd(c.X, w1[:, :, :H], w1[:, :, H:], w2, "silu", off)[3]
    _, _, _, rX, r1g, r1u, r2 = O.glu_bwd(g, c.X, z[:, :H], z[:, H:], w1[:, :, :H], w1[:, :, H:], w2, "silu", off)
    for got, want, what in ((Y, y, "Y"), (Yserve, y, "Y, nothing kept"), (dX, rX, "dX"), (dW1, np.concatenate((r1g, r1u), 2), "dW1"), (dW2, r2, "dW2")):
        err = np.abs(base.host(got) - want).max()
        assert err <= tol * np.abs(want).max(), (what, err, np.abs(want).max())


# few rows, tiles of 128 and of 256
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ns,behind,K,N", [((5, 9, 0, 1), 3, 520, 136), ((200, 0, 145, 9), 6, 136, 272), ((1300, 257), 4, 72, 8200)])
@pytest.mark.parametrize("bad", BAD)
def test_products_from_four_bits(ns, behind, K, N, dtype, bad):
    c, hole = holes(ns, behind, K, N, dtype, bad)
    W = c.stored(c.rng.standard_normal((c.E, K, N)) / np.sqrt(K))
    xq, xs = store(c.x.view(1, *c.x.shape), False)
    Wq, Ws = store(W, True)
    Y = c.fresh(c.R, N)
    api.moe_ragged_gemm_mx4(xq, xs, c.S, c.inv, c.k, Wq, Ws, c.off, c.R, c.E, K, N, Y)
    assert (Y[:c.offsets[-1]][torch.from_numpy(hole[:c.offsets[-1]])] == 0).all()
    x, w = four_bits.kept(c.X), np.stack([four_bits.kept(m.T).T for m in base.host(W)])
    ref = O.gemm(x, w, c.offsets)
    base.check(Y, ref, c.half * np.abs(ref) + (1 + c.half) * c.sums(K) * O.gemm(np.abs(x), np.abs(w), c.offsets), "Y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ns,behind,M,H", [((5, 9, 0, 1), 3, 520, 136), ((200, 0, 145, 9), 6, 136, 272), ((1300, 257), 4, 72, 4104)])
@pytest.mark.parametrize("bad", BAD)
def test_glu_from_four_bits(ns, behind, M, H, dtype, bad):
    c, hole = holes(ns, behind, M, H, dtype, bad)
    n = c.offsets[-1]
    W1 = c.stored(c.rng.standard_normal((c.E, M, 2 * H)) / np.sqrt(M))
    W2 = c.stored(c.rng.standard_normal((c.E, H, M)) / np.sqrt(H))
    (W1q, W1s), (W2q, W2s) = store(W1, True), store(W2, True)
    Y, clean = c.fresh(c.R, M), c.fresh(c.R, M)
    ws = torch.empty(api.moe_ragged_glu_mx4_workspace_bytes(c.S, c.R, c.E, M, H), dtype=torch.uint8, device=DEV)
    call = lambda x, y: api.moe_ragged_glu_mx4(x, c.S, c.inv, c.k, W1q, W1s, W2q, W2s, c.off, c.R, c.E, M, H, api.MOE_ACT_SILU, y, ws)
    call(c.x, Y)
    assert (Y[:n][torch.from_numpy(hole[:n])] == 0).all()
    x = c.x.clone()
    x[0] = 0                                      # nobody asks for it: the same bits as with a token of zeros
    call(x, clean)
    assert torch.equal(Y, clean) and torch.isfinite(Y).all()
