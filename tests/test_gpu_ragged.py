"""GPU parity: the plan of ragged rows, the products over them and the expert FFN with its 8-bit pre-activation, against the float64
checker, element by element.

Bounds.  A sum of K products carries at most K 2^-23 of the sum of magnitudes in fp32 (a matrix instruction may truncate; the products'
own rounding in fp32 is inside that), in fp64, which forms the pre-activation that is kept from fp32 operands, K 2^-50.  bf16 stores round by 2^-8 of the value, fp32 stores by 2^-24.  The bf16
activation is a polynomial off by 6e-5 and its derivative by 1e-4; in fp32 both are erf's, off by 2^-21 (1 + |z|).  Each bound below
carries these through the products that follow, in magnitudes."""
import numpy as np
import pytest
import torch

from oracle import ragged_oracle as O
from paper_2407_00599_amd import api
from util import DEV, torch_dtype

pytestmark = pytest.mark.gpu


def host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def check(got, ref, bound, what):
    got = host(got)
    err = np.abs(got - ref)
    bad = ~(err <= bound + 1e-30)
    assert not bad.any(), (what, int(bad.sum()), tuple(int(v[0]) for v in np.nonzero(bad)), float(err[bad].max()), float((err / (bound + 1e-30))[bad].max()))


def routing(rng, S, k, E, C, shares=None):
    """idx, slot, counts of a gate: shares skews the experts, an expert with share 0 gets no row."""
    p = np.ones(E) if shares is None else np.asarray(shares, float)
    idx = np.stack([rng.choice(E, k, replace=False, p=p / p.sum()) for _ in range(S)]).astype(np.int32)
    counts, slot = np.zeros(E, np.int32), np.full((S, k), -1, np.int32)
    for j in range(k):
        for t in range(S):
            e = idx[t, j]
            if counts[e] < C:
                slot[t, j] = counts[e]
            counts[e] += 1
    return idx, slot, counts


def run_plan(idx, slot, counts, S, E, k, C):
    i32 = lambda *s: torch.full(s, -9, dtype=torch.int32, device=DEV)
    d = lambda a: torch.from_numpy(a).to(DEV)
    off, ri, rs, inv = i32(E + 1), i32(S, k), i32(S, k), i32(k, S)
    api.moe_ragged_plan(d(idx), d(slot), d(counts), S, E, k, C, off, ri, rs, inv)
    return off, ri, rs, inv


@pytest.mark.parametrize("S,k,E,C", [(1, 1, 1, 1), (1, 2, 8, 1), (5, 3, 3, 5), (64, 2, 8, 64), (300, 2, 256, 300), (333, 4, 7, 90),
                                     (1000, 2, 3, 10), (257, 8, 70, 257)])
def test_plan(S, k, E, C):
    rng = np.random.default_rng(S + E)
    idx, slot, counts = routing(rng, S, k, E, C)
    off, ri, rs, inv = run_plan(idx, slot, counts, S, E, k, C)
    offsets, row, rinv = O.plan(idx, slot, counts, C)
    assert np.array_equal(host(off), offsets)
    assert np.array_equal(host(inv).reshape(-1), rinv)
    got = host(ri).astype(np.int64) * S + host(rs)
    assert np.array_equal(np.where(host(rs) < 0, -1, got), row)
    assert (host(ri)[row < 0] == 0).all() and (host(rs)[row < 0] == -1).all()


class Case:
    """Rows with given numbers per expert; `behind` rows at the end belong to none.  gather: rows of a token matrix through a map."""

    def __init__(self, ns, behind, K, N, dtype, gather, seed):
        rng = self.rng = np.random.default_rng(seed)
        self.dtype, self.t = dtype, torch_dtype(dtype)
        self.half = torch.finfo(self.t).eps / 2
        self.E, self.R = len(ns), sum(ns) + behind
        self.offsets = np.concatenate([[0], np.cumsum(ns)])
        self.off = torch.from_numpy(self.offsets.astype(np.int32)).to(DEV)
        self.k = 3 if gather else 1
        self.S = -(-self.R // self.k) if gather else 0
        self.K, self.N = K, N
        x = self.stored(rng.standard_normal((self.S if gather else self.R, K)))
        self.x = x
        self.inv = None
        if gather:
            inv = np.full(self.R, -1, np.int32)
            inv[:self.offsets[-1]] = rng.permutation(self.S * self.k)[:self.offsets[-1]]
            self.inv = torch.from_numpy(inv).to(DEV)
            self.X = O.rows_of(host(x), inv, self.k)
        else:
            self.X = host(x)
        self.live = np.arange(self.R)[:, None] < self.offsets[-1]

    def stored(self, a):
        return torch.from_numpy(np.ascontiguousarray(a)).to(self.t).to(DEV)

    def fresh(self, *shape, fill=7.0):
        return torch.full(shape, fill, dtype=self.t, device=DEV)

    def sums(self, K, kept=False):       # what a sum of K products may be off by, of its magnitudes
        return K * 2.0 ** (-50 if kept and self.dtype == "f32" else -23)

    def source(self):
        return self.x, self.S, self.inv, self.k


PRODUCTS = [
    ((1,), 0, 8, 8, True), ((1, 0), 1, 64, 128, True), ((0, 0, 3), 2, 72, 40, False), ((5, 0, 17, 64, 1), 4, 264, 136, True),
    ((33, 31, 32, 64, 65), 0, 128, 256, True), ((0,), 9, 64, 64, False), ((200, 0, 55), 70, 520, 328, True),
    ((300, 513), 1, 72, 1032, False), ((1,) * 70 + (0,) * 10 + (4,) * 20, 3, 64, 72, True), ((130, 257, 5, 0), 200, 1040, 264, True),
    ((700, 900), 0, 256, 2048, True), ((2,) * 8, 0, 1024, 512, True),
    # few weights over many rows: reductions in parts, one of them of an expert without rows
    ((4000,), 5, 64, 136, True), ((2000, 0, 2900), 0, 128, 72, False),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ns,behind,K,N,gather", PRODUCTS)
def test_products(ns, behind, K, N, gather, dtype):
    c = Case(ns, behind, K, N, dtype, gather, 3 * K + N)
    W = c.stored(c.rng.standard_normal((c.E, K, N)) / np.sqrt(K))
    dY = c.stored(c.rng.standard_normal((c.R, N)))
    ws = torch.empty(max(api.moe_ragged_gemm_workspace_bytes(api.dtype_code(c.x), c.R, c.E, K, N),
                         api.moe_ragged_gemm_workspace_bytes(api.dtype_code(c.x), c.R, c.E, N, K),
                         api.moe_ragged_wgrad_workspace_bytes(api.dtype_code(c.x), c.R, c.E, K, N), 16), dtype=torch.uint8, device=DEV)
    w, g = host(W), host(dY)
    args = c.source()
    Y = c.fresh(c.R, N)
    api.moe_ragged_gemm(*args, W, 0, c.off, c.R, c.E, K, N, Y, ws)
    ref = O.gemm(c.X, w, c.offsets)
    check(Y, ref, c.half * np.abs(ref) + c.sums(K) * O.gemm(np.abs(c.X), np.abs(w), c.offsets), "Y")
    Wt = W.transpose(1, 2).contiguous()
    Y2 = c.fresh(c.R, N)
    api.moe_ragged_gemm(*args, Wt, 1, c.off, c.R, c.E, K, N, Y2, ws)
    check(Y2, ref, c.half * np.abs(ref) + c.sums(K) * O.gemm(np.abs(c.X), np.abs(w), c.offsets), "Y of W^T")
    dX = c.fresh(c.R, K)
    api.moe_ragged_gemm(dY, 0, None, 1, W, 1, c.off, c.R, c.E, N, K, dX, ws)
    wt = w.transpose(0, 2, 1)
    ref = O.gemm(g, wt, c.offsets)
    check(dX, ref, c.half * np.abs(ref) + c.sums(N) * O.gemm(np.abs(g), np.abs(wt), c.offsets), "dX")
    dW = c.fresh(c.E, K, N)
    api.moe_ragged_wgrad(*args, dY, c.off, c.R, c.E, K, N, dW, ws)
    ref = O.wgrad(c.X, g, c.offsets)
    check(dW, ref, c.half * np.abs(ref) + c.sums(max(ns) + 1) * O.wgrad(np.abs(c.X), np.abs(g), c.offsets), "dW")


def test_rows_of_other_experts_do_not_leak():
    """Infinities and NaN in an expert's rows, in rows behind the last expert and in tokens that no row asks for stay where they are."""
    for dtype in ("f32", "bf16"):
        c = Case((40, 3, 70), 30, 136, 72, dtype, True, 5)
        inv = host(c.inv)
        c.x[inv[45] // c.k] = float("inf")                    # a row of expert 2 (and of whoever shares the token)
        unused = sorted(set(range(c.S)) - set(inv[:113] // c.k))
        c.x[unused] = float("nan")
        bad = np.isin(inv[:113] // c.k, [inv[45] // c.k])
        W = c.stored(c.rng.standard_normal((3, 136, 72)))
        dY = c.stored(c.rng.standard_normal((c.R, 72)))
        dY[113:] = float("nan")
        Y, dX, dW = c.fresh(c.R, 72), c.fresh(c.R, 136), c.fresh(3, 136, 72)
        ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
        api.moe_ragged_gemm(*c.source(), W, 0, c.off, c.R, 3, 136, 72, Y, ws)
        api.moe_ragged_gemm(dY, 0, None, 1, W, 1, c.off, c.R, 3, 72, 136, dX, ws)
        api.moe_ragged_wgrad(*c.source(), dY, c.off, c.R, 3, 136, 72, dW, ws)
        finite = np.isfinite(host(Y)).all(1)
        assert np.array_equal(~finite[:113], bad) and (host(Y)[113:] == 0).all()
        assert np.isfinite(host(dX)).all() and (host(dX)[113:] == 0).all()
        owns = [bad[a:b].any() for a, b in zip(c.offsets[:-1], c.offsets[1:])]
        assert [not np.isfinite(v).all() for v in host(dW)] == owns


FFN = [   # rows per expert, rows behind, M, H, n_esp, esp_idx, gather
    ((1,), 0, 64, 64, 1, 0, True), ((2, 0, 1), 1, 64, 128, 1, 0, True), ((20, 0, 45, 9), 6, 136, 272, 2, 1, True),
    ((64, 33, 0, 100), 0, 72, 1032, 1, 0, False), ((150, 70), 40, 264, 520, 1, 0, True), ((3,) * 66, 0, 64, 40, 1, 0, True),
    ((400, 90, 513), 30, 128, 768, 4, 2, True), ((12,) * 8, 0, 512, 1024, 1, 0, True),
    ((2100, 0, 2600), 20, 64, 72, 1, 0, True), ((3200,), 0, 72, 136, 1, 0, False),     # weight gradients in parts
    # few rows of large experts: a row, an expert with more rows than go along with one reading, experts without any, a shard
    ((1,), 0, 512, 2048, 1, 0, True), ((0, 3, 0, 0, 1, 0, 7, 0), 3, 520, 2200, 1, 0, True), ((40, 0, 1, 0, 2, 0, 0), 5, 512, 4160, 2, 1, True),
    ((20,), 2, 264, 4096, 1, 0, False), ((0,) * 65 + (3, 0, 2), 1, 136, 8200, 1, 0, True),
]


def kept_is_near(q, s, z, dz, what):
    """The kept form of z, which is known to +-dz: the scale of a magnitude in that range, and the nearest whole number."""
    rows, cols = z.shape
    for n in range(s.shape[1]):
        b = slice(32 * n, min(32 * n + 32, cols))
        lo, hi = (np.abs(z[:, b]) - dz[:, b]).max(1), (np.abs(z[:, b]) + dz[:, b]).max(1)
        for r in range(rows):
            assert O.scale_byte(max(lo[r], 0.0)) <= s[r, n] <= O.scale_byte(hi[r]), (what, r, n)
        step = np.exp2(s[:, n:n + 1].astype(float) - 133)
        assert (np.abs(q[:, b] * step - z[:, b]) <= step / 2 + dz[:, b]).all(), (what, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ns,behind,M,H,n_esp,esp_idx,gather", FFN)
def test_ffn(ns, behind, M, H, n_esp, esp_idx, gather, dtype):
    c = Case(ns, behind, M, H, dtype, gather, M + H)
    Hl = H // n_esp
    h = slice(esp_idx * Hl, (esp_idx + 1) * Hl)
    W1 = c.stored(c.rng.standard_normal((c.E, M, H)) / np.sqrt(M))
    W2 = c.stored(c.rng.standard_normal((c.E, H, M)) / np.sqrt(Hl))
    w1, w2 = host(W1)[:, :, h], host(W2)[:, h]
    code, R, E, off = api.dtype_code(c.x), c.R, c.E, c.offsets
    nz = (Hl + 31) // 32
    A, Y, Yserve = c.fresh(R, Hl), c.fresh(R, M), c.fresh(R, M)
    Zq = torch.full((R, Hl), 99, dtype=torch.int8, device=DEV)
    Zs = torch.full((R, nz), 99, dtype=torch.uint8, device=DEV)
    ws = torch.empty(max(api.moe_ragged_ffn_workspace_bytes(code, R, E, M, H, n_esp, b) for b in (0, 1)) + 16, dtype=torch.uint8, device=DEV)
    shape = (c.off, R, E, M, H, esp_idx, n_esp)
    api.moe_ragged_ffn_fwd(*c.source(), W1, W2, *shape, Zq, Zs, A, Y, ws)
    api.moe_ragged_ffn_fwd(*c.source(), W1, W2, *shape, None, None, c.fresh(R, Hl), Yserve, ws)
    z = O.gemm(c.X, w1, off)
    dz = c.sums(M) * O.gemm(np.abs(c.X), np.abs(w1), off)
    a = O.gelu(z)
    act = 6e-5 if dtype == "bf16" else 2.0 ** -21 * (1 + np.abs(z))
    da = c.half * np.abs(a) + (1 + c.half) * (act + 1.13 * dz)        # |GeLU'| < 1.13
    y = O.gemm(a, w2, off)
    by = O.gemm(da, np.abs(w2), off) + c.sums(Hl) * O.gemm(np.abs(a) + da, np.abs(w2), off)
    for got, what in ((Y, "Y"), (Yserve, "Y, nothing kept")):
        check(got, y, by + c.half * (np.abs(y) + by), what)
    n = off[-1]
    dkept = c.sums(M, kept=True) * O.gemm(np.abs(c.X), np.abs(w1), off)
    kept_is_near(host(Zq)[:n].astype(float), host(Zs)[:n], z[:n], dkept[:n] + 2.0 ** -50 * np.abs(z[:n]), "kept")
    assert (host(Zq)[n:] == 99).all() and (host(Zs)[n:] == 99).all()

    # backward, from the checker's kept form; rows behind the last expert hold NaN blocks, which nothing may read
    q, s = O.store8(z)
    z = O.load8(q, s)
    s[n:] = 255
    Zq, Zs = torch.from_numpy(q).to(DEV), torch.from_numpy(s).to(DEV)
    dY = c.stored(c.rng.standard_normal((R, M)))
    dY[n:] = float("nan")
    g = host(dY)
    g[n:] = 0
    dX, dW1, dW2 = c.fresh(R, M), c.fresh(E, M, H), c.fresh(E, H, M)
    api.moe_ragged_ffn_bwd(dY, *c.source(), Zq, Zs, W1, W2, *shape, dX, dW1, dW2, ws)
    rX, r1, r2 = O.ffn_bwd(g, c.X, z, w1, w2, off)
    w2t, w1t = w2.transpose(0, 2, 1), w1.transpose(0, 2, 1)
    dA = O.gemm(g, w2t, off)
    bA = c.sums(M) * O.gemm(np.abs(g), np.abs(w2t), off)
    dgrad = 1e-4 if dtype == "bf16" else 2.0 ** -20 * (1 + np.abs(z))
    gr = np.abs(O.gelu_grad(z))
    dZ = dA * O.gelu_grad(z)
    bZ = bA * (gr + dgrad) + np.abs(dA) * dgrad + 2.0 ** -23 * np.abs(dZ)
    bZ = bZ + c.half * (np.abs(dZ) + bZ)
    act = 6e-5 if dtype == "bf16" else 2.0 ** -21 * (1 + np.abs(z))
    a = O.gelu(z)
    bact = act + c.half * (np.abs(a) + act)
    mag = np.abs(dZ) + bZ
    bX = O.gemm(bZ, np.abs(w1t), off) + c.sums(Hl) * O.gemm(mag, np.abs(w1t), off)
    check(dX, rX, bX + c.half * (np.abs(rX) + bX), "dX")
    rows = c.sums(max(ns) + 1)
    b1 = O.wgrad(np.abs(c.X), bZ, off) + rows * O.wgrad(np.abs(c.X), mag, off)
    check(dW1[:, :, h], r1, b1 + c.half * (np.abs(r1) + b1), "dW1")
    b2 = O.wgrad(bact, np.abs(g), off) + rows * O.wgrad(np.abs(a) + bact, np.abs(g), off)
    check(dW2[:, h], r2, b2 + c.half * (np.abs(r2) + b2), "dW2")
    # of the whole weight gradients only the shard's part is written
    dW1[:, :, h], dW2[:, h] = 7, 7
    assert (dW1 == 7).all() and (dW2 == 7).all()


def test_not_finite_pre_activations():
    """A row with an infinity keeps NaN blocks; the other rows' gradients do not see it."""
    c = Case((5, 4), 0, 64, 96, "bf16", False, 11)
    c.x[2, 3] = float("inf")
    W1, W2 = c.stored(c.rng.standard_normal((2, 64, 96))), c.stored(c.rng.standard_normal((2, 96, 64)))
    Zq, Zs = torch.empty(9, 96, dtype=torch.int8, device=DEV), torch.empty(9, 3, dtype=torch.uint8, device=DEV)
    ws = torch.empty(api.moe_ragged_ffn_workspace_bytes(api.MOE_BF16, 9, 2, 64, 96, 1, 1), dtype=torch.uint8, device=DEV)
    Y, dX, dW1, dW2 = c.fresh(9, 64), c.fresh(9, 64), c.fresh(2, 64, 96), c.fresh(2, 96, 64)
    api.moe_ragged_ffn_fwd(*c.source(), W1, W2, c.off, 9, 2, 64, 96, 0, 1, Zq, Zs, c.fresh(9, 96), Y, None)
    api.moe_ragged_ffn_bwd(c.stored(np.ones((9, 64))), *c.source(), Zq, Zs, W1, W2, c.off, 9, 2, 64, 96, 0, 1, dX, dW1, dW2, ws)
    assert (host(Zs)[2] == 255).all() and (np.delete(host(Zs), 2, 0) != 255).all()
    for t in (Y, dX):
        finite = np.isfinite(host(t)).all(1)
        assert not finite[2] and np.delete(finite, 2).all()
    assert np.isfinite(host(dW1)[1]).all() and np.isfinite(host(dW2)[1]).all() and not np.isfinite(host(dW2)[0]).all()


def test_on_another_stream():
    """Work goes to the current stream: a call behind a slow copy on a side stream sees what the copy wrote."""
    c = Case((600, 500), 0, 512, 512, "bf16", False, 13)
    W = c.stored(c.rng.standard_normal((2, 512, 512)) / 20)
    Y, ref = c.fresh(c.R, 512), c.fresh(c.R, 512)
    api.moe_ragged_gemm(*c.source(), W, 0, c.off, c.R, 2, 512, 512, ref, None)
    torch.cuda.synchronize()
    late = torch.zeros_like(c.x)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(50):
            late.zero_()
        late.copy_(c.x)
        api.moe_ragged_gemm(late, 0, None, 1, W, 0, c.off, c.R, 2, 512, 512, Y, None)
    side.synchronize()
    assert torch.equal(Y, ref)
