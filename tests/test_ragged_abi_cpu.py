"""Refusals of the dropless block's entry points: everything is rejected on the host before a launch.  And the polynomial that the
ragged FFN's epilogues evaluate is the fitted one."""
import ctypes
import importlib.util
import os
import re

import numpy as np
import pytest

from paper_2407_00599_amd import api

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_00599_amd", "csrc")
A = ctypes.c_void_p(0x1000)        # aligned dummy pointers: never dereferenced on these paths
U = ctypes.c_void_p(0x1004)        # misaligned
BIG = 1 << 60
EINVAL, EUNSUPPORTED, EALIGN, EWORKSPACE, ENULL = -1, -2, -3, -5, -6


@pytest.fixture(scope="module")
def L():
    return api.lib()


def test_plan_refusals(L):
    def call(idx=A, slot=A, counts=A, S=16, E=4, k=2, C=16, off=A, ri=A, rs=A, inv=A):
        return L.moe_ragged_plan(idx, slot, counts, S, E, k, C, off, ri, rs, inv, None)
    for kw in ({"S": 0}, {"E": 0}, {"k": 0}, {"k": 5}, {"C": 0}):
        assert call(**kw) == EINVAL, kw
    for kw in ({"E": 257}, {"k": 9, "E": 16}, {"S": 1 << 30, "k": 1}, {"S": 1 << 28, "k": 3, "C": 4}):
        assert call(**kw) == EUNSUPPORTED, kw
    for n in ("idx", "slot", "counts", "off", "ri", "rs", "inv"):
        assert call(**{n: None}) == ENULL and call(**{n: U}) == EALIGN, n


def test_product_refusals(L):
    def gemm(x=A, dt=1, S=16, inv=A, k=2, W=A, tr=0, off=A, R=32, E=4, K=64, N=128, Y=A, ws=A, wsb=BIG):
        return L.moe_ragged_gemm(x, dt, S, inv, k, W, tr, off, R, E, K, N, Y, ws, wsb, None)

    def wgrad(x=A, dt=1, S=16, inv=A, k=2, W=A, off=A, R=32, E=4, K=64, N=128, Y=A, ws=A, wsb=BIG):
        return L.moe_ragged_wgrad(x, dt, S, inv, k, W, off, R, E, K, N, Y, ws, wsb, None)
    for f in (gemm, wgrad):
        for kw in ({"dt": 2}, {"dt": -1}, {"R": 0}, {"E": 0}, {"K": 0}, {"N": -8}, {"S": 0}, {"k": 0}, {"inv": None}):   # rows as they lie: k = 1
            assert f(**kw) == EINVAL, (f, kw)
        for kw in ({"E": 257}, {"K": 60}, {"N": 12}, {"k": 9}, {"R": (1 << 29) + 1, "K": 8, "N": 8}, {"R": 1 << 20, "N": 4096},
                   {"S": 1 << 29}, {"S": 1 << 26, "K": 64}, {"K": 1 << 20, "N": 4096, "R": 8, "S": 8},
                   {"dt": 0, "R": 1 << 29, "N": 4096}):
            assert f(**kw) == EUNSUPPORTED, (f, kw)
        for n in ("x", "W", "off", "Y"):
            assert f(**{n: None}) == ENULL and f(**{n: U}) == EALIGN, (f, n)
        assert f(inv=U) == EALIGN
    assert gemm(tr=2) == EINVAL and gemm(tr=-1) == EINVAL


def test_ffn_refusals(L):
    w = L.moe_ragged_ffn_workspace_bytes
    need = w(1, 32, 4, 64, 256, 2, 1)
    assert need >= 2 * 32 * 128 * 2
    for bad in ((2, 32, 4, 64, 256, 2), (1, 0, 4, 64, 256, 2), (1, 32, 4, 64, 255, 2), (1, 32, 4, 60, 256, 2)):
        assert w(*bad, 1) == 0 and w(*bad, 0) == 0

    def fwd(x=A, dt=1, S=16, inv=A, k=2, W1=A, W2=A, off=A, R=32, E=4, M=64, H=256, e=0, n=2, Zq=A, Zs=A, Act=A, Y=A, ws=A, wsb=BIG):
        return L.moe_ragged_ffn_fwd(x, dt, S, inv, k, W1, W2, off, R, E, M, H, e, n, Zq, Zs, Act, Y, ws, wsb, None)

    def bwd(dY=A, x=A, dt=1, S=16, inv=A, k=2, Zq=A, Zs=A, W1=A, W2=A, off=A, R=32, E=4, M=64, H=256, e=0, n=2, dX=A, dW1=A, dW2=A,
            ws=A, wsb=need):
        return L.moe_ragged_ffn_bwd(dY, x, dt, S, inv, k, Zq, Zs, W1, W2, off, R, E, M, H, e, n, dX, dW1, dW2, ws, wsb, None)
    for f in (fwd, bwd):
        for kw in ({"dt": 5}, {"R": 0}, {"E": 0}, {"M": 0}, {"H": 0}, {"H": 255}, {"e": 2}, {"e": -1}, {"n": 0}, {"S": 0}, {"k": 0},
                   {"inv": None}):
            assert f(**kw) == EINVAL, (f, kw)
        for kw in ({"E": 300}, {"M": 60}, {"H": 264}, {"k": 9}, {"R": 1 << 25, "H": 512}, {"S": 1 << 28, "k": 3}):
            assert f(**kw) == EUNSUPPORTED, (f, kw)
    for n in ("x", "W1", "W2", "off", "Act", "Y"):
        assert fwd(**{n: None}) == ENULL and fwd(**{n: U}) == EALIGN, n
    assert fwd(Zq=None) == ENULL and fwd(Zs=None) == ENULL        # both or neither
    assert fwd(Zq=U) == EALIGN and fwd(Zs=U) == EALIGN
    for n in ("dY", "x", "Zq", "Zs", "W1", "W2", "off", "dX", "dW1", "dW2"):
        assert bwd(**{n: None}) == ENULL and bwd(**{n: U}) == EALIGN, n
    assert bwd(ws=None) == EWORKSPACE and bwd(wsb=64) == EWORKSPACE and bwd(ws=U) == EALIGN


def test_ckpt8_refusals(L):
    for f in (lambda x=A, dt=1, r=4, c=64, q=A, s=A: L.moe_ckpt8_store(x, dt, r, c, q, s, None),
              lambda x=A, dt=1, r=4, c=64, q=A, s=A: L.moe_ckpt8_load(q, s, r, c, x, dt, None)):
        assert f(dt=2) == EINVAL and f(r=0) == EINVAL and f(c=0) == EINVAL and f(c=20) == EUNSUPPORTED
        for n in ("x", "q", "s"):
            assert f(**{n: None}) == ENULL and f(**{n: U}) == EALIGN, n


def test_norm_refusals(L):
    LAYER, RMS = api.MOE_NORM_LAYER, api.MOE_NORM_RMS
    need = L.moe_norm_bwd_workspace_bytes(100, 64)
    assert L.moe_norm_bwd_workspace_bytes(0, 64) == 0 and L.moe_norm_bwd_workspace_bytes(4, 60) == 0

    def fwd(x=A, dt=1, S=100, M=64, kind=LAYER, w=A, b=A, eps=1e-5, u=A, mean=A, rstd=A):
        return L.moe_norm_fwd(x, dt, S, M, kind, w, b, eps, u, mean, rstd, None)

    def res(h=A, x=A, dt=1, S=100, M=64, kind=LAYER, w=A, b=A, gate=A, gk=1, alpha=1.0, eps=1e-5, y=A, mean=A, rstd=A):
        return L.moe_norm_residual_fwd(h, x, dt, S, M, kind, w, b, gate, gk, alpha, eps, y, mean, rstd, None)

    def bwd(du=A, x=A, dt=1, S=100, M=64, kind=LAYER, w=A, mean=A, rstd=A, dres=A, dx=A, dw=A, db=A, ws=A, wsb=need):
        return L.moe_norm_bwd(du, x, dt, S, M, kind, w, mean, rstd, dres, dx, dw, db, ws, wsb, None)

    def resb(dy=A, h=A, dt=1, S=100, M=64, kind=LAYER, w=A, b=A, gate=A, gk=1, alpha=1.0, mean=A, rstd=A, dh=A, dw=A, db=A, dg=A,
             ws=A, wsb=need):
        return L.moe_norm_residual_bwd(dy, h, dt, S, M, kind, w, b, gate, gk, alpha, mean, rstd, dh, dw, db, dg, ws, wsb, None)
    for f in (fwd, res, bwd, resb):
        for kw in ({"dt": 3}, {"S": 0}, {"M": 0}, {"kind": 2}, {"kind": -1}):
            assert f(**kw) == EINVAL, (f, kw)
        assert f(M=60) == EUNSUPPORTED and f(M=32776) == EUNSUPPORTED
        assert f(w=None) == ENULL and f(w=U) == EALIGN
        assert f(kind=RMS) == EINVAL                                # a bias or a mean has no place in it
    for f in (fwd, res):
        assert f(eps=-1.0) == EINVAL and f(eps=float("nan")) == EINVAL
        assert f(x=None) == ENULL and f(mean=U) == EALIGN and f(rstd=U) == EALIGN
    for f in (res, resb):
        assert f(gk=3) == EINVAL and f(gate=None) == ENULL and f(gk=0) == EINVAL
    assert resb(gate=None, gk=0) == EINVAL                          # dgate without a gate
    for f in (bwd, resb):
        assert f(mean=None) == ENULL and f(rstd=None) == ENULL and f(dw=None) == ENULL
        assert need > 0 and f(ws=None) == EWORKSPACE and f(wsb=need - 1) == EWORKSPACE and f(ws=U) == EALIGN
    assert bwd(dres=U) == EALIGN and bwd(dx=None) == ENULL and resb(dh=None) == ENULL and resb(dg=U) == EALIGN


def test_binding_refuses_mixed_types():
    import torch
    f, h, i = torch.zeros(8), torch.zeros(8, dtype=torch.bfloat16), torch.zeros(8, dtype=torch.int64)
    with pytest.raises(ValueError):
        api.moe_ragged_gemm(f, 0, None, 1, h, 0, torch.zeros(2, dtype=torch.int32), 1, 1, 8, 8, f)
    with pytest.raises(ValueError):
        api.moe_ragged_plan(i, i, i, 1, 1, 1, 1, i, i, i, i)
    with pytest.raises(ValueError):
        api.moe_ckpt8_store(f, 1, 8, i, torch.zeros(1, dtype=torch.uint8))      # the 8-bit values are int8
    with pytest.raises(ValueError):
        api.moe_norm_fwd(h, 1, 8, api.MOE_NORM_RMS, h, None, 1e-5, h)     # weights are fp32


def test_polynomial_is_the_fitted_one():
    spec = importlib.util.spec_from_file_location("fit_gelu_poly", os.path.join(CSRC, "fit_gelu_poly.py"))
    fit = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(fit)
    body = re.search(r"PHI_ODD\[\d+\] = \{([^}]*)\}", open(os.path.join(CSRC, "ragged.h")).read()).group(1)
    table = np.array([float(t.strip().rstrip("f")) for t in body.split(",")], dtype=np.float32)
    np.testing.assert_allclose(table, fit.tables()[0], rtol=2e-6)
