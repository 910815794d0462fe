"""GPU parity of the ragged products and of the ragged FFN in the tiles that large problems take: each size below is the smallest around
which the dispatch chooses the tile that is named beside it, with a narrow reduction so that the checker keeps up.  The tests themselves, their
checker and their bounds are those of test_gpu_ragged.py; the 8-bit forms of whole tensors come from eight_bits.py."""
import numpy as np
import pytest
import torch

import eight_bits
import test_gpu_ragged as base
from oracle import ragged_oracle as O
from paper_2407_00599_amd import api
from util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def whole_tensors(monkeypatch):
    monkeypatch.setattr(base.O, "store8", eight_bits.store8)
    monkeypatch.setattr(base, "kept_is_near", eight_bits.kept_is_near)


# rows per expert, rows behind, K, N, gather
PRODUCTS = [
    ((700, 0, 830), 20, 72, 8200, True),       # 256 x 256, weight gradient 256 x 256
    ((1010, 3, 12), 5, 72, 8200, False),       # 192 x 256
    ((300, 220), 0, 72, 8200, True),           # 128 x 128
    ((50, 1, 0, 149), 10, 64, 4104, True),     # 64 x 64
]


@pytest.mark.parametrize("ns,behind,K,N,gather", PRODUCTS)
def test_products(ns, behind, K, N, gather):
    base.test_products(ns, behind, K, N, gather, "bf16")


# rows per expert, rows behind, M, H, n_esp, esp_idx, gather: the tile of the two launches that form and read the 8-bit values
FFN = [
    ((700, 0, 830), 20, 72, 8200, 1, 0, True),               # 256 x 256
    ((1010, 3, 12), 5, 72, 16400, 2, 1, True),               # 192 x 256, a shard
    ((300, 220), 0, 72, 8200, 1, 0, False),                  # 128 x 128
    ((50, 1, 0, 149), 10, 64, 4104, 1, 0, True),             # 64 x 64
    # the merged backward launch with dX in these tiles beside weight gradients of 256 x 256
    ((900, 1200, 0, 900), 10, 4104, 72, 1, 0, True),         # 256 x 256
    ((1300, 2, 500, 190), 8, 4104, 72, 1, 0, True),          # 192 x 256
    ((300, 0, 0, 695), 5, 4104, 72, 1, 0, True),             # 128 x 128
]


@pytest.mark.parametrize("ns,behind,M,H,n_esp,esp_idx,gather", FFN)
def test_ffn(ns, behind, M, H, n_esp, esp_idx, gather):
    base.test_ffn(ns, behind, M, H, n_esp, esp_idx, gather, "bf16")


def test_ffn_f32_kept_in_large_tiles():
    """64 x 64 tiles on the fp64 matrix cores, full of rows"""
    base.test_ffn((450, 0, 350), 6, 72, 4104, 1, 0, True, "f32")


def test_few_rows_over_many_experts():
    """Few rows over so many experts that the second product has more tiles than workgroups: no parts, and a workgroup takes a second tile."""
    E, M, H, S, k = 66, 1032, 2064, 32, 2
    rng = np.random.default_rng(4)
    ns = np.ones(E, np.int64)
    ns[[3, 4, 11, 30, 64, 65]], ns[7] = 0, 4
    n, R = int(ns.sum()), S * k
    assert n < R <= 64 and int((ns > 0).sum()) * -(-M // 128) > 512
    assert api.moe_ragged_ffn_workspace_bytes(api.MOE_BF16, R, E, M, H, 1, 0) > 0       # of the kernels for few rows
    offsets = np.concatenate([[0], np.cumsum(ns)])
    inv = np.full(R, -1, np.int32)
    inv[:n] = rng.permutation(R)[:n]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(5)
    normal = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    x = normal(S, M).bfloat16()
    W1, W2 = (normal(E, M, H) / M ** 0.5).bfloat16(), (normal(E, H, M) / H ** 0.5).bfloat16()
    off = torch.from_numpy(offsets.astype(np.int32)).to(DEV)
    dinv = torch.from_numpy(inv).to(DEV)
    A = torch.full((R, H), 7.0, dtype=torch.bfloat16, device=DEV)
    Y = torch.full((R, M), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.full((api.moe_ragged_ffn_workspace_bytes(api.MOE_BF16, R, E, M, H, 1, 0),), 0x55, dtype=torch.uint8, device=DEV)
    api.moe_ragged_ffn_fwd(x, S, dinv, k, W1, W2, off, R, E, M, H, 0, 1, None, None, A, Y, ws)
    X = torch.from_numpy(O.rows_of(base.host(x), inv, k)).to(DEV)
    half, sums = 2.0 ** -8, 2.0 ** -23      # as in test_gpu_ragged.py
    for e in range(E):
        r = slice(int(offsets[e]), int(offsets[e + 1]))
        if r.start == r.stop:
            continue
        w1, w2 = W1[e].double(), W2[e].double()
        z, dz = X[r] @ w1, M * sums * (X[r].abs() @ w1.abs())
        a = z * 0.5 * torch.erfc(-z / 2 ** 0.5)
        da = half * a.abs() + (1 + half) * (6e-5 + 1.13 * dz)
        y = a @ w2
        by = da @ w2.abs() + H * sums * ((a.abs() + da) @ w2.abs())
        bound = by + half * (y.abs() + by)
        err = (Y[r].double() - y).abs()
        assert (err <= bound).all(), (e, float((err / bound).max()))
    assert (Y[n:] == 0).all()


def test_calls_of_several_launches_on_a_side_stream():
    """Every launch of a call goes to the current stream: behind slow work on a side stream, whose result is the call's input, calls of
    several launches see what it wrote, and the default stream is not waited for."""
    c = base.Case((5, 0, 9, 4), 2, 512, 2048, "bf16", True, 17)
    big = base.Case((4000,), 0, 64, 136, "bf16", False, 18)
    bf = lambda *s: c.stored(c.rng.standard_normal(s))
    W1, W2 = c.stored(c.rng.standard_normal((4, 512, 2048)) / 23), c.stored(c.rng.standard_normal((4, 2048, 512)) / 45)
    dY, dyb = bf(c.R, 512), bf(4000, 136)
    S, M = 600, 512
    h, dy = bf(S, M), bf(S, M)
    f32 = lambda *s: torch.empty(*s, device=DEV)
    w = torch.ones(M, device=DEV)
    rstd = torch.full((S,), 0.9, device=DEV)
    code = api.MOE_BF16
    ws = torch.empty(max(api.moe_ragged_ffn_workspace_bytes(code, c.R, 4, 512, 2048, 1, 0), api.moe_ragged_ffn_workspace_bytes(code, c.R, 4, 512, 2048, 1, 1),
                         api.moe_ragged_wgrad_workspace_bytes(code, 4000, 1, 64, 136), api.moe_norm_bwd_workspace_bytes(S, M)), dtype=torch.uint8, device=DEV)
    A = c.fresh(c.R, 2048)
    Zq, Zs = torch.empty(c.R, 2048, dtype=torch.int8, device=DEV), torch.empty(c.R, 64, dtype=torch.uint8, device=DEV)

    def calls(x, xb, hh):
        out = {n: c.fresh(*s) for n, s in (("serve", (c.R, 512)), ("Y", (c.R, 512)), ("dX", (c.R, 512)), ("dW1", (4, 512, 2048)),
                                           ("dW2", (4, 2048, 512)), ("dW", (1, 64, 136)), ("dh", (S, M)))}
        out["dw"] = f32(M)
        shape = (W1, W2, c.off, c.R, 4, 512, 2048, 0, 1)
        api.moe_ragged_ffn_fwd(x, c.S, c.inv, c.k, *shape, None, None, A, out["serve"], ws)
        api.moe_ragged_ffn_fwd(x, c.S, c.inv, c.k, *shape, Zq, Zs, A, out["Y"], ws)
        api.moe_ragged_ffn_bwd(dY, x, c.S, c.inv, c.k, Zq, Zs, *shape, out["dX"], out["dW1"], out["dW2"], ws)
        api.moe_ragged_wgrad(xb, 0, None, 1, dyb, big.off, 4000, 1, 64, 136, out["dW"], ws)
        api.moe_norm_residual_bwd(dy, hh, S, M, api.MOE_NORM_RMS, w, None, None, api.MOE_GATE_NONE, 0.5, None, rstd, out["dh"], out["dw"],
                                  None, None, ws)
        return out
    ref = calls(c.x, big.x, h)
    late = [torch.zeros_like(t) for t in (c.x, big.x, h)]
    load = torch.randn(4096, 4096, device=DEV) / 64
    torch.cuda.synchronize()                  # the zeros are written, on whichever stream
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(20):                   # some 20 ms
            load = load @ load
        for to, src in zip(late, (c.x, big.x, h)):
            to.copy_(src)
        got = calls(*late)
    side.synchronize()
    for n in ref:
        assert torch.equal(got[n], ref[n]), n
