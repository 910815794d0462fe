"""GPU: rows among an expert's own whose map entry names no token (negative, or past the last one) are rows of zeros, forward and backward,
also where token 0, which stands in for them, is not finite."""
import numpy as np
import pytest
import torch

import eight_bits
import test_gpu_ragged as base
from oracle import ragged_oracle as O
from paper_2407_00599_amd import api
from util import DEV

pytestmark = pytest.mark.gpu


def holes(ns, behind, M, H, dtype, bad):
    """A case whose every fifth row or so names no token, and whose token 0 is not finite and asked for by nobody else."""
    c = base.Case(ns, behind, M, H, dtype, True, M + H)
    inv, n = base.host(c.inv).copy(), int(c.offsets[-1])
    hole = np.zeros(c.R, bool)
    hole[:n:5] = True
    hole[:n] |= inv[:n] < c.k                                # whoever had token 0
    inv[:n][hole[:n]] = np.resize([-1, c.S * c.k, -7, c.S * c.k + 1000], int(hole.sum()))
    c.inv = torch.from_numpy(inv.astype(np.int32)).to(DEV)
    c.x[0] = bad
    tokens = np.where(hole | (inv < 0), 0, inv // c.k)
    c.X = np.where((hole | (inv < 0))[:, None], 0.0, base.host(c.x)[tokens])
    assert hole[:n].any() and np.isfinite(c.X).all()
    return c, hole


# sizes that take the small tiles (few rows in serving), 192 x 256 and 256 x 256
@pytest.mark.parametrize("dtype,ns,behind,M,H", [
    ("f32", (20, 0, 45, 9), 6, 136, 272), ("bf16", (20, 0, 45, 9), 6, 136, 272), ("bf16", (5, 9, 0, 1), 3, 520, 2200),
    ("bf16", (1010, 3, 12), 5, 72, 8200), ("bf16", (700, 0, 830), 20, 72, 8200)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_ffn(dtype, ns, behind, M, H, bad):
    c, hole = holes(ns, behind, M, H, dtype, bad)
    E, R, off = c.E, c.R, c.offsets
    n = off[-1]
    W1 = c.stored(c.rng.standard_normal((E, M, H)) / np.sqrt(M))
    W2 = c.stored(c.rng.standard_normal((E, H, M)) / np.sqrt(H))
    dY = c.stored(c.rng.standard_normal((R, M)))
    A, Y, Yserve, dX = c.fresh(R, H), c.fresh(R, M), c.fresh(R, M), c.fresh(R, M)
    dW1, dW2 = c.fresh(E, M, H), c.fresh(E, H, M)
    Zq = torch.full((R, H), 99, dtype=torch.int8, device=DEV)
    Zs = torch.full((R, (H + 31) // 32), 99, dtype=torch.uint8, device=DEV)
    ws = torch.empty(max(api.moe_ragged_ffn_workspace_bytes(api.dtype_code(c.x), R, E, M, H, 1, b) for b in (0, 1)) + 16, dtype=torch.uint8, device=DEV)
    shape = (c.off, R, E, M, H, 0, 1)
    api.moe_ragged_ffn_fwd(*c.source(), W1, W2, *shape, None, None, c.fresh(R, H), Yserve, ws)
    api.moe_ragged_ffn_fwd(*c.source(), W1, W2, *shape, Zq, Zs, A, Y, ws)
    api.moe_ragged_ffn_bwd(dY, *c.source(), Zq, Zs, W1, W2, *shape, dX, dW1, dW2, ws)
    for t in (A, Y, Yserve):
        assert (t[:n][torch.from_numpy(hole[:n])] == 0).all()
    assert (Zq[:n][torch.from_numpy(hole[:n])] == 0).all() and (Zs[:n][torch.from_numpy(hole[:n])] == 0).all()
    # the other rows and the gradients are those of a token matrix that holds zeros there: tolerance of the tensors as a whole, 2^-6 for six
    # roundings of 2^-8 in bf16 whose errors add up like their squares, a thousandth of that for fp32's 2^-24
    tol = 2.0 ** -6 if dtype == "bf16" else 2.0 ** -16
    w1, w2, g = base.host(W1), base.host(W2), base.host(dY)
    g[n:] = 0
    z = O.gemm(c.X, w1, off)
    y = O.gemm(O.gelu(z), w2, off)
    z = O.load8(base.host(Zq), base.host(Zs))
    z[n:] = 0
    rX, r1, r2 = O.ffn_bwd(g, c.X, z, w1, w2, off)
    for got, want, what in ((Y, y, "Y"), (Yserve, y, "Y, nothing kept"), (dX, rX, "dX"), (dW1, r1, "dW1"), (dW2, r2, "dW2")):
        err = np.abs(base.host(got) - want).max()
        assert err <= tol * np.abs(want).max(), (what, err, np.abs(want).max())


def test_kept_form_of_a_row_without_a_token_is_that_of_zeros():
    """Also where token 0 is finite: scale byte 0, as moe_ckpt8_store keeps a row of zeros."""
    c, hole = holes((40, 3, 21), 4, 64, 96, "bf16", 1.0)
    W1, W2 = c.stored(c.rng.standard_normal((3, 64, 96))), c.stored(c.rng.standard_normal((3, 96, 64)))
    Zq, Zs = torch.empty(c.R, 96, dtype=torch.int8, device=DEV), torch.empty(c.R, 3, dtype=torch.uint8, device=DEV)
    api.moe_ragged_ffn_fwd(*c.source(), W1, W2, c.off, c.R, 3, 64, 96, 0, 1, Zq, Zs, c.fresh(c.R, 96), c.fresh(c.R, 64), None)
    zero = eight_bits.store8(np.zeros((1, 96)))
    n = c.offsets[-1]
    assert (base.host(Zq)[:n][hole[:n]] == zero[0]).all() and (base.host(Zs)[:n][hole[:n]] == zero[1]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ns,behind,K,N", [((20, 0, 45, 9), 6, 136, 272), ((700, 0, 830), 20, 72, 8200), ((2100, 1900), 5, 64, 136)])
def test_products(ns, behind, K, N, dtype):
    c, hole = holes(ns, behind, K, N, dtype, float("nan"))
    E, R, off = c.E, c.R, c.offsets
    n = off[-1]
    W, dY = c.stored(c.rng.standard_normal((E, K, N)) / np.sqrt(K)), c.stored(c.rng.standard_normal((R, N)))
    Y, dW = c.fresh(R, N), c.fresh(E, K, N)
    code = api.dtype_code(c.x)
    ws = torch.empty(max(api.moe_ragged_gemm_workspace_bytes(code, R, E, K, N), api.moe_ragged_wgrad_workspace_bytes(code, R, E, K, N), 16),
                     dtype=torch.uint8, device=DEV)
    api.moe_ragged_gemm(*c.source(), W, 0, c.off, R, E, K, N, Y, ws)
    api.moe_ragged_wgrad(*c.source(), dY, c.off, R, E, K, N, dW, ws)
    w, g = base.host(W), base.host(dY)
    g[n:] = 0
    ref, refw = O.gemm(c.X, w, off), O.wgrad(c.X, g, off)
    base.check(Y, ref, c.half * np.abs(ref) + c.sums(K) * O.gemm(np.abs(c.X), np.abs(w), off), "Y")
    base.check(dW, refw, c.half * np.abs(refw) + c.sums(max(ns) + 1) * O.wgrad(np.abs(c.X), np.abs(g), off), "dW")
    assert (Y[:n][torch.from_numpy(hole[:n])] == 0).all()
