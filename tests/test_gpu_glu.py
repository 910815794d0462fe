"""GPU parity of the gated expert FFN over ragged rows, forward, kept values and backward, against the float64 oracle, element by element.

Bounds.  Sums as in test_gpu_ragged.py: K 2^-23 of the sum of magnitudes in fp32.  bf16 stores round by 2^-8 of the value, fp32 stores by 2^-24.
The bf16 GeLU is a polynomial off by 6e-5, its derivative by 1e-4; SiLU uses an exponential, a reciprocal and, in
fp32, a divide, each within 2^-22, of an argument rounded by 2^-24 of |g| log2(e): 2^-21 (1 + |g|) of |g| covers the value and 2^-20 (1 + |g|)^2 the
slope, whose own terms are g s (1 - s) and s.  In fp32 the GeLU's are those of test_gpu_ragged.py.  Slopes of both are under 1.13."""
import numpy as np
import pytest
import torch

from oracle import ragged_oracle as O
from paper_2407_00599_amd import api
from test_gpu_ragged import Case, check, host
from util import DEV

pytestmark = pytest.mark.gpu
CODE = {"silu": api.MOE_ACT_SILU, "gelu": api.MOE_ACT_GELU}


def act_bounds(act, dtype, g):
    """how far act(g) and act'(g) may be off"""
    g = np.abs(g)
    if act == "silu":
        return 2.0 ** -21 * (1 + g) * g + 1e-30, 2.0 ** -20 * (1 + g) ** 2
    if dtype == "bf16":
        return np.full_like(g, 6e-5), np.full_like(g, 1e-4)
    return 2.0 ** -21 * (1 + g), 2.0 ** -20 * (1 + g)


class Glu:
    """A shard's weights beside a Case's rows"""

    def __init__(self, ns, behind, M, H, n_esp, esp_idx, gather, dtype):
        c = self.c = Case(ns, behind, M, H, dtype, gather, M + 2 * H)
        Hl = self.Hl = H // n_esp
        self.gate = slice(esp_idx * Hl, (esp_idx + 1) * Hl)
        self.up = slice(H + esp_idx * Hl, H + (esp_idx + 1) * Hl)
        self.W1 = c.stored(c.rng.standard_normal((c.E, M, 2 * H)) * 1.5 / np.sqrt(M))
        self.W2 = c.stored(c.rng.standard_normal((c.E, H, M)) / np.sqrt(Hl))
        w1 = host(self.W1)
        self.wg, self.wu, self.w2 = w1[:, :, self.gate], w1[:, :, self.up], host(self.W2)[:, self.gate]
        self.shape = (c.off, c.R, c.E, M, H, esp_idx, n_esp)
        code = api.dtype_code(c.x)
        self.ws = torch.empty(max(api.moe_ragged_glu_workspace_bytes(code, c.R, c.E, M, H, n_esp, b) for b in (0, 1)) + 16, dtype=torch.uint8, device=DEV)


# rows per expert, rows behind, M, H, n_esp, esp_idx, gather
SIZES = [
    ((1,), 0, 8, 8, 1, 0, True), ((1,), 0, 64, 64, 1, 0, False), ((2, 0, 1), 1, 64, 128, 1, 0, True), ((0, 0), 3, 64, 64, 1, 0, True),
    ((20, 0, 45, 9), 6, 136, 272, 2, 1, True), ((64, 33, 0, 100), 0, 72, 1032, 1, 0, False), ((150, 70), 40, 264, 520, 1, 0, True),
    ((3,) * 66, 0, 64, 40, 1, 0, True), ((400, 90, 513), 30, 128, 768, 4, 2, True), ((12,) * 8, 0, 512, 1024, 1, 0, True),
    ((7, 30), 0, 72, 48, 2, 1, False),                                                 # a shard of 24 columns: the halves meet inside a k tile
    ((2100, 0, 2600), 20, 64, 72, 1, 0, True), ((3200,), 0, 72, 136, 1, 0, False),     # weight gradients in parts
    # few rows of large experts: a row, an expert with more rows than go along with one reading, experts without any, a shard
    ((1,), 0, 512, 2048, 1, 0, True), ((0, 3, 0, 0, 1, 0, 7, 0), 3, 520, 2200, 1, 0, True), ((40, 0, 1, 0, 2, 0, 0), 5, 512, 4160, 2, 1, True),
    ((20,), 2, 264, 4096, 1, 0, False), ((0,) * 65 + (3, 0, 2), 1, 136, 8200, 1, 0, True),
]
# few rows of large experts (bf16), in the kernels for them
FEW = [
    ((3, 0, 9, 1, 0, 2, 17, 4), 5, 264, 4096, 1, 0, True),   # 128 hidden columns a workgroup, an expert with more rows than go along with one reading
    ((5, 20, 0), 2, 520, 5400, 1, 0, True),                  # 64 hidden columns
    ((20, 9), 1, 520, 16400, 2, 1, False),                   # two groups of rows, a shard, rows as they lie
    ((0, 0, 31, 1), 0, 1032, 2072, 1, 0, True),
]
# the tiles of large problems (bf16), each around the smallest size for which the dispatch chooses it
LARGE = [
    ((700, 0, 830), 20, 72, 4104, 1, 0, True),               # forward 256 x 256, gradients of g and u 128 x 128
    ((1010, 3, 12), 5, 72, 8208, 2, 1, True),                # 192 x 256, 128 x 128, a shard
    ((700, 0, 830), 20, 72, 8200, 1, 0, False),              # 256 x 256, 256 x 256
    ((1010, 3, 12), 5, 72, 16400, 2, 1, True),               # 192 x 256, 192 x 256, a shard
    ((50, 1, 0, 149), 10, 64, 4104, 1, 0, True),             # 64 x 128, 64 x 64
    ((130, 257, 5, 0), 200, 1040, 2064, 1, 0, True),         # 64 x 128, 64 x 128
    # the merged backward launch with dX in these tiles beside weight gradients of 256 x 256
    ((900, 1200, 0, 900), 10, 4104, 72, 1, 0, True),         # 256 x 256
    ((1300, 2, 500, 190), 8, 4104, 144, 2, 1, True),         # 256 x 256, a shard
    ((5000, 4200, 4100, 3300), 8, 4104, 72, 1, 0, False),    # 256 x 256, weight gradients of many k tiles
    ((300, 0, 0, 695), 5, 4104, 72, 1, 0, False),            # 128 x 128
]


def run(size, dtype, act):
    ns, M, H = size[0], size[2], size[3]
    s = Glu(*size, dtype)
    c, Hl = s.c, s.Hl
    R, E, off, n = c.R, c.E, c.offsets, c.offsets[-1]
    A, Y, Yserve, Z = c.fresh(R, Hl), c.fresh(R, M), c.fresh(R, M), c.fresh(R, 2 * Hl)
    api.moe_ragged_glu_fwd(*c.source(), s.W1, s.W2, *s.shape, CODE[act], Z, A, Y, s.ws)
    api.moe_ragged_glu_fwd(*c.source(), s.W1, s.W2, *s.shape, CODE[act], None, c.fresh(R, Hl), Yserve, s.ws)
    G, U, a, y = O.glu_fwd(c.X, s.wg, s.wu, s.w2, act, off)
    X = np.abs(c.X)
    dG, dU = c.sums(M) * O.gemm(X, np.abs(s.wg), off), c.sums(M) * O.gemm(X, np.abs(s.wu), off)
    for got, ref, d, what in ((Z[:n, :Hl], G, dG, "G"), (Z[:n, Hl:], U, dU, "U")):
        check(got, ref[:n], (d + c.half * (np.abs(ref) + d))[:n], what)
    assert (host(Z)[n:] == 7).all() and (host(A)[n:] == 7).all()
    ea, _ = act_bounds(act, dtype, np.abs(G) + dG)
    va = np.abs(O.gate_act(act, G)[0])
    ea = ea + 1.13 * dG
    bA = ea * (np.abs(U) + dU) + va * dU + 2.0 ** -23 * np.abs(a)
    bA = bA + c.half * (np.abs(a) + bA)
    bY = O.gemm(bA, np.abs(s.w2), off) + c.sums(Hl) * O.gemm(np.abs(a) + bA, np.abs(s.w2), off)
    for got, what in ((Y, "Y"), (Yserve, "Y, nothing kept")):
        check(got, y, bY + c.half * (np.abs(y) + bY), what)

    # backward, at the kept values; rows behind the last expert hold NaN, which nothing may read
    g, u = host(Z)[:, :Hl], host(Z)[:, Hl:]
    g[n:] = u[n:] = 0
    Z[n:] = float("nan")
    dY = c.stored(c.rng.standard_normal((R, M)))
    dY[n:] = float("nan")
    gy = host(dY)
    gy[n:] = 0
    dX, dW1, dW2 = c.fresh(R, M), c.fresh(E, M, 2 * H), c.fresh(E, H, M)
    api.moe_ragged_glu_bwd(dY, *c.source(), Z, s.W1, s.W2, *s.shape, CODE[act], dX, dW1, dW2, s.ws)
    rG, rU, ra, rX, r1g, r1u, r2 = O.glu_bwd(gy, c.X, g, u, s.wg, s.wu, s.w2, act, off)
    w2t = s.w2.transpose(0, 2, 1)
    dA, bdA = O.gemm(gy, w2t, off), c.sums(M) * O.gemm(np.abs(gy), np.abs(w2t), off)
    ea, es = act_bounds(act, dtype, g)
    va, vs = (np.abs(v) for v in O.gate_act(act, g))

    def product(ref, *factors):            # of values known to +- their bounds, rounded in fp32 twice and stored
        full = size_ = 1.0
        for v, b in factors:
            full, size_ = full * (np.abs(v) + b), size_ * np.abs(v)
        b = full - size_ + 2.0 ** -22 * full
        return b + c.half * (np.abs(ref) + b)
    exact = np.zeros_like(u)
    bG, bU = product(rG, (dA, bdA), (u, exact), (vs, es)), product(rU, (dA, bdA), (va, ea))
    ba = product(ra, (va, ea), (u, exact))
    wgt, wut = s.wg.transpose(0, 2, 1), s.wu.transpose(0, 2, 1)
    both = lambda p, q: O.gemm(p, np.abs(wgt), off) + O.gemm(q, np.abs(wut), off)
    bX = both(bG, bU) + c.sums(2 * Hl) * both(np.abs(rG) + bG, np.abs(rU) + bU)
    check(dX, rX, bX + c.half * (np.abs(rX) + bX), "dX")
    rows = c.sums(max(ns) + 1)
    for got, ref, left, bl, mag, what in ((dW1[:, :, s.gate], r1g, X, bG, np.abs(rG) + bG, "dW1, gate"), (dW1[:, :, s.up], r1u, X, bU, np.abs(rU) + bU, "dW1, up")):
        b = O.wgrad(left, bl, off) + rows * O.wgrad(left, mag, off)
        check(got, ref, b + c.half * (np.abs(ref) + b), what)
    b = O.wgrad(ba, np.abs(gy), off) + rows * O.wgrad(np.abs(ra) + ba, np.abs(gy), off)
    check(dW2[:, s.gate], r2, b + c.half * (np.abs(r2) + b), "dW2")
    # of the whole weight gradients only the shard's part is written
    dW1[:, :, s.gate], dW1[:, :, s.up], dW2[:, s.gate] = 7, 7, 7
    assert (dW1 == 7).all() and (dW2 == 7).all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: f"{sum(s[0])}x{s[2]}x{s[3]}")
def test_glu(size, dtype, act):
    run(size, dtype, act)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("size", FEW, ids=lambda s: f"{sum(s[0])}x{s[2]}x{s[3]}")
def test_glu_of_few_rows(size, act):
    ns, behind, M, H, n_esp = size[:5]
    R, E = sum(ns) + behind, len(ns)
    tiles = api.moe_ragged_glu_workspace_bytes(api.MOE_BF16, 65, E, M, H, n_esp, 0)      # no parts in bf16
    assert api.moe_ragged_glu_workspace_bytes(api.MOE_BF16, R, E, M, H, n_esp, 0) > tiles == 0
    run(size, "bf16", act)


@pytest.mark.parametrize("size", LARGE, ids=lambda s: f"{sum(s[0])}x{s[2]}x{s[3]}")
def test_glu_in_large_tiles(size):
    run(size, "bf16", "silu")


def test_a_dense_gated_block():
    """One expert with all rows, as they lie, against automatic differentiation."""
    R, M, H = 70, 64, 96
    gen = torch.Generator().manual_seed(3)
    n = lambda *s: torch.randn(*s, generator=gen).to(DEV)
    x, W1, W2, dY = n(R, M), n(1, M, 2 * H) / 8, n(1, H, M) / 10, n(R, M)
    off = torch.tensor([0, R], dtype=torch.int32, device=DEV)
    A, Y, Z, dX, dW1, dW2 = (torch.empty(*s, device=DEV) for s in ((R, H), (R, M), (R, 2 * H), (R, M), (1, M, 2 * H), (1, H, M)))
    ws = torch.empty(api.moe_ragged_glu_workspace_bytes(api.MOE_F32, R, 1, M, H, 1, 1), dtype=torch.uint8, device=DEV)
    api.moe_ragged_glu_fwd(x, 0, None, 1, W1, W2, off, R, 1, M, H, 0, 1, api.MOE_ACT_SILU, Z, A, Y, ws)
    api.moe_ragged_glu_bwd(dY, x, 0, None, 1, Z, W1, W2, off, R, 1, M, H, 0, 1, api.MOE_ACT_SILU, dX, dW1, dW2, ws)
    leaves = [t.detach().cpu().double().requires_grad_() for t in (x, W1, W2)]
    z = leaves[0] @ leaves[1][0]
    y = (torch.nn.functional.silu(z[:, :H]) * z[:, H:]) @ leaves[2][0]
    y.backward(dY.cpu().double())
    for got, ref in zip((Y, dX, dW1, dW2), (y.detach(), *(t.grad for t in leaves))):
        # K 2^-23 of sums of magnitudes that are some sqrt(K) times the results' size, through three products
        assert float((got.cpu().double() - ref).abs().max() / ref.abs().max()) < 3 * 96 * 2.0 ** -23


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_other_experts_do_not_leak(dtype):
    """An infinity in a token and NaN in an expert's weights stay in the rows and gradients that they belong to."""
    s = Glu((40, 3, 70), 30, 136, 72, 1, 0, True, dtype)
    c = s.c
    inv = host(c.inv)
    c.x[inv[45] // c.k] = float("inf")
    bad = np.isin(inv[:113] // c.k, [inv[45] // c.k])
    s.W1[1, 5, 70] = float("nan")
    bad[40:43] = True
    Z, Y, dX = c.fresh(c.R, 144), c.fresh(c.R, 136), c.fresh(c.R, 136)
    dW1, dW2 = c.fresh(3, 136, 144), c.fresh(3, 72, 136)
    dY = c.stored(c.rng.standard_normal((c.R, 136)))
    api.moe_ragged_glu_fwd(*c.source(), s.W1, s.W2, *s.shape, CODE["silu"], Z, c.fresh(c.R, 72), Y, s.ws)
    api.moe_ragged_glu_bwd(dY, *c.source(), Z, s.W1, s.W2, *s.shape, CODE["silu"], dX, dW1, dW2, s.ws)
    for t in (Y, dX):
        finite = np.isfinite(host(t)).all(1)
        assert np.array_equal(~finite[:113], bad) and (host(t)[113:] == 0).all()
    owns = [bad[a:b].any() for a, b in zip(c.offsets[:-1], c.offsets[1:])]
    assert [not np.isfinite(v).all() for v in host(dW1)] == owns and [not np.isfinite(v).all() for v in host(dW2)] == owns


def test_same_bits_again_and_from_a_graph():
    """Both passes, with reductions in parts, repeated and replayed: no result depends on an order of arrival."""
    s = Glu((2100, 0, 2600), 20, 64, 72, 1, 0, True, "bf16")
    c = s.c
    out = {n: c.fresh(*v) for n, v in {"Z": (c.R, 144), "A": (c.R, 72), "Y": (c.R, 64), "dX": (c.R, 64), "dW1": (3, 64, 144), "dW2": (3, 72, 64)}.items()}
    dY = c.stored(c.rng.standard_normal((c.R, 64)))

    def step():
        api.moe_ragged_glu_fwd(*c.source(), s.W1, s.W2, *s.shape, CODE["silu"], out["Z"], out["A"], out["Y"], s.ws)
        api.moe_ragged_glu_bwd(dY, *c.source(), out["Z"], s.W1, s.W2, *s.shape, CODE["silu"], out["dX"], out["dW1"], out["dW2"], s.ws)
    step()
    torch.cuda.synchronize()
    ref = {n: t.clone() for n, t in out.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for n, t in out.items():
            t[:4700] = -3
        s.ws.fill_(255)                                     # what the workspace held before does not matter
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n, t in out.items():
            assert torch.equal(t, ref[n]), n
        step()
        torch.cuda.synchronize()
