"""GPU parity: norms in front of and behind a block, forward and backward, against the float64 checker.

Bounds.  A sum of a row is formed by at most 32 additions in a thread, 6 or 4 exchanges and up to 16 partial sums: under 64 fp32
roundings, 2^-18 of the sum of magnitudes.  So a centred value is off by 2^-18 mean|v| + 2^-24 of itself, a normalised one by 2^-17 of
big = |hat| + rstd mean|v| (the statistics' own rounding included), and everything linear in it by 2^-17 to 2^-16 of the same
expression in magnitudes.  A column sum over S rows adds (S + 64) 2^-24 of its magnitudes.  The storage type's half step comes on top."""
import numpy as np
import pytest
import torch

from oracle import ragged_oracle as O
from paper_2407_00599_amd import api
from util import DEV, torch_dtype

pytestmark = pytest.mark.gpu
EPS = 1e-5
F32 = np.float32

# every number of threads to a row and pieces to a thread; one row, odd numbers of rows, rows that end inside a piece's turn
SHAPES = [(1, 8), (1, 4096), (3, 64), (37, 128), (100, 136), (65, 512), (9, 1024), (50, 1544), (33, 2048), (70, 2056), (5, 4096),
          (3, 8192), (2, 12000), (2, 32768), (3000, 72), (700, 520)]


def make(S, M, dtype, offset, seed):
    rng = np.random.default_rng(seed)
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(torch_dtype(dtype)).to(DEV)
    f = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=F32)).to(DEV)
    n = rng.standard_normal
    return {"x": d(n((S, M)) * 2 + offset), "h": d(n((S, M)) + 0.25 - offset), "du": d(n((S, M))), "dy": d(n((S, M))),
            "w": f(1 + 0.1 * n(M)), "b": f(0.1 * n(M)), "gate_channel": f(rng.random(M)), "gate_token": f(rng.random(S))}


def host(t):
    return t.double().cpu().numpy()


def check(got, ref, bound, what):
    got = host(got)
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(np.abs(got - ref)[bad].max()), float((np.abs(got - ref) / bound)[bad].max()))


def stats(v, mean, rstd, hat):
    return np.abs(hat) + rstd[:, None] * np.abs(v).mean(1, keepdims=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("S,M", SHAPES)
def test_in_front(S, M, kind, dtype):
    layer, half = kind == "layer", torch.finfo(torch_dtype(dtype)).eps / 2
    t = make(S, M, dtype, 30.0 if M == 512 else 0.0, S + M)      # (once with a mean far from zero)
    K = api.MOE_NORM_LAYER if layer else api.MOE_NORM_RMS
    b = t["b"] if layer else None
    u = torch.full_like(t["x"], 9)
    mean, rstd = (torch.full((S,), 9.0, device=DEV) for _ in range(2))
    api.moe_norm_fwd(t["x"], S, M, K, t["w"], b, EPS, u, mean if layer else None, rstd)
    x, w, du, dres = host(t["x"]), host(t["w"]), host(t["du"]), host(t["dy"])
    bb = host(b) if layer else None
    ref, rm, rr, hat = O.norm(x, w, bb, EPS, layer)
    big = stats(x, rm, rr, hat)
    check(u, ref, half * np.abs(ref) + 2.0 ** -17 * (big * np.abs(w) + np.abs(bb if layer else 0)) + 1e-30, "u")
    check(rstd, rr, 2.0 ** -17 * rr * (1 + (rr * np.abs(x).mean(1)) * np.abs(hat).mean(1)), "rstd")
    if layer:
        check(mean, rm, 2.0 ** -18 * np.abs(x).mean(1) + 1e-30, "mean")
    u2 = torch.full_like(u, 9)
    api.moe_norm_fwd(t["x"], S, M, K, t["w"], b, EPS, u2)        # nothing kept for a backward pass
    assert torch.equal(u, u2)
    # backward, from the checker's statistics
    mean, rstd = (torch.from_numpy(v.astype(F32)).to(DEV) for v in (rm, rr))
    ws = torch.empty(max(api.moe_norm_bwd_workspace_bytes(S, M), 16), dtype=torch.uint8, device=DEV)
    for res in (t["dy"], None):
        dx = torch.full_like(t["x"], 9)
        dw, db = (torch.full((M,), 9.0, device=DEV) for _ in range(2))
        api.moe_norm_bwd(t["du"], t["x"], S, M, K, t["w"], mean if layer else None, rstd, res, dx, dw, db if layer else None, ws)
        hat = (x - (host(mean)[:, None] if layer else 0)) * host(rstd)[:, None]
        dv, rw, rb = O.norm_grad(du, hat, host(rstd), w, layer)
        rdx = dv + (dres if res is not None else 0)
        gw = np.abs(du * w)
        inner = gw + big * (gw * big).mean(1, keepdims=True) + gw.mean(1, keepdims=True)
        check(dx, rdx, half * np.abs(rdx) + 2.0 ** -16 * rr[:, None] * inner + 2.0 ** -23 * np.abs(dres), "dx")
        cols = 2.0 ** -16 + (S + 64) * 2.0 ** -24
        check(dw, rw, cols * (np.abs(du) * big).sum(0), "dw")
        if layer:
            check(db, rb, cols * np.abs(du).sum(0), "db")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("S,M", SHAPES)
def test_behind(S, M, gate, kind, dtype):
    layer, half, alpha = kind == "layer", torch.finfo(torch_dtype(dtype)).eps / 2, float(F32(0.3))
    t = make(S, M, dtype, 30.0 if M == 512 else 0.0, 7 * S + M)
    K = api.MOE_NORM_LAYER if layer else api.MOE_NORM_RMS
    gk = {"none": api.MOE_GATE_NONE, "channel": api.MOE_GATE_CHANNEL, "token": api.MOE_GATE_TOKEN}[gate]
    b, g = (t["b"] if layer else None), (None if gate == "none" else t["gate_" + gate])
    y = torch.full_like(t["x"], 9)
    mean, rstd = (torch.full((S,), 9.0, device=DEV) for _ in range(2))
    api.moe_norm_residual_fwd(t["h"], t["x"], S, M, K, t["w"], b, g, gk, alpha, EPS, y, mean if layer else None, rstd)
    h, x, w, dy = (host(t[n]) for n in ("h", "x", "w", "dy"))
    bb, gg = (host(b) if layer else None), (None if g is None else host(g))
    ref, rm, rr, hat, n = O.norm_residual(h, x, w, bb, gg, gate, alpha, EPS, layer)
    big, sg = stats(h, rm, rr, hat), O.spread_gate(gg, gate)
    nbig = big * np.abs(w) + np.abs(bb if layer else 0)
    check(y, ref, half * np.abs(ref) + 2.0 ** -16 * alpha * sg * nbig + 2.0 ** -23 * np.abs(x), "y")
    mean, rstd = (torch.from_numpy(v.astype(F32)).to(DEV) for v in (rm, rr))
    hat = (h - (host(mean)[:, None] if layer else 0)) * host(rstd)[:, None]
    n = hat * w + (bb if layer else 0)
    ws = torch.empty(max(api.moe_norm_bwd_workspace_bytes(S, M), 16), dtype=torch.uint8, device=DEV)
    dh = torch.full_like(t["h"], 9)
    dw, db = (torch.full((M,), 9.0, device=DEV) for _ in range(2))
    dg = None if g is None else torch.full_like(g, 9)
    api.moe_norm_residual_bwd(t["dy"], t["h"], S, M, K, t["w"], b, g, gk, alpha, mean if layer else None, rstd, dh, dw,
                              db if layer else None, dg, ws)
    rdh, rw, rb, rg = O.norm_residual_grad(dy, n, hat, host(rstd), w, gg, gate, alpha, layer)
    up = np.abs(alpha * sg * dy)
    gw = up * np.abs(w)
    inner = gw + big * (gw * big).mean(1, keepdims=True) + gw.mean(1, keepdims=True)
    check(dh, rdh, half * np.abs(rdh) + 2.0 ** -16 * rr[:, None] * inner + 1e-30, "dh")
    cols = 2.0 ** -16 + (S + 64) * 2.0 ** -24
    check(dw, rw, cols * (up * big).sum(0) + 1e-30, "dw")
    if layer:
        check(db, rb, cols * up.sum(0) + 1e-30, "db")
    if g is not None:
        each = np.abs(alpha * dy) * nbig
        check(dg, rg, (2.0 ** -16 * each.sum(1) if gate == "token" else cols * each.sum(0)) + 1e-30, "dgate")
        # a second run gives the same bits
        dw2, dg2 = torch.full_like(dw, 9), torch.full_like(dg, 9)
        api.moe_norm_residual_bwd(t["dy"], t["h"], S, M, K, t["w"], b, g, gk, alpha, mean if layer else None, rstd, dh, dw2, None, dg2, ws)
        assert torch.equal(dw, dw2) and torch.equal(dg, dg2)


def test_a_row_that_is_not_finite_stays_alone():
    S, M = 6, 256
    t = make(S, M, "f32", 0.0, 1)
    t["x"][2, 7] = float("inf")
    t["x"][4, 9] = float("nan")
    t["x"][5] = 0
    u = torch.empty_like(t["x"])
    api.moe_norm_fwd(t["x"], S, M, api.MOE_NORM_RMS, t["w"], None, EPS, u)
    ok = [0, 1, 3]
    ref = O.norm(host(t["x"])[ok], host(t["w"]), None, EPS, False)[0]
    assert np.abs(host(u)[ok] - ref).max() < 1e-4
    assert torch.isnan(u[4]).all() and torch.isnan(u[2, 7]) and (u[5] == 0).all()
