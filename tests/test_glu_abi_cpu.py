"""Refusals of the gated FFN's entry points: everything is rejected on the host before a launch.  And the oracle's gradients against
differences."""
import ctypes

import numpy as np
import pytest

from oracle import ragged_oracle as O
from paper_2407_00599_amd import api

A = ctypes.c_void_p(0x1000)        # aligned dummy pointers: never dereferenced on these paths
U = ctypes.c_void_p(0x1004)        # misaligned
BIG = 1 << 60
EINVAL, EUNSUPPORTED, EALIGN, EWORKSPACE, ENULL = -1, -2, -3, -5, -6


def test_glu_refusals():
    L = api.lib()
    w = L.moe_ragged_glu_workspace_bytes
    need = w(1, 32, 4, 64, 256, 2, 1)
    assert need >= 3 * 32 * 128 * 2
    for bad in ((2, 32, 4, 64, 256, 2), (1, 0, 4, 64, 256, 2), (1, 32, 4, 64, 255, 2), (1, 32, 4, 60, 256, 2), (1, 32, 4, 64, 1 << 29, 2)):
        assert w(*bad, 1) == 0 and w(*bad, 0) == 0

    def fwd(x=A, dt=1, S=16, inv=A, k=2, W1=A, W2=A, off=A, R=32, E=4, M=64, H=256, e=0, n=2, act=0, Z=A, Act=A, Y=A, ws=A, wsb=BIG):
        return L.moe_ragged_glu_fwd(x, dt, S, inv, k, W1, W2, off, R, E, M, H, e, n, act, Z, Act, Y, ws, wsb, None)

    def bwd(dY=A, x=A, dt=1, S=16, inv=A, k=2, Z=A, W1=A, W2=A, off=A, R=32, E=4, M=64, H=256, e=0, n=2, act=0, dX=A, dW1=A, dW2=A,
            ws=A, wsb=need):
        return L.moe_ragged_glu_bwd(dY, x, dt, S, inv, k, Z, W1, W2, off, R, E, M, H, e, n, act, dX, dW1, dW2, ws, wsb, None)
    for f in (fwd, bwd):
        for kw in ({"dt": 5}, {"R": 0}, {"E": 0}, {"M": 0}, {"H": 0}, {"H": 255}, {"e": 2}, {"e": -1}, {"n": 0}, {"S": 0}, {"k": 0},
                   {"inv": None}, {"act": 2}, {"act": -1}):
            assert f(**kw) == EINVAL, (f, kw)
        for kw in ({"E": 300}, {"M": 60}, {"H": 264}, {"k": 9}, {"R": 1 << 25, "H": 256}, {"S": 1 << 28, "k": 3}, {"H": 1 << 29},
                   {"M": 1 << 15, "H": 1 << 16, "R": 8, "S": 8}):
            assert f(**kw) == EUNSUPPORTED, (f, kw)
    for n in ("x", "W1", "W2", "off", "Act", "Y"):
        assert fwd(**{n: None}) == ENULL and fwd(**{n: U}) == EALIGN, n
    assert fwd(Z=U) == EALIGN and fwd(ws=U) == EALIGN and fwd(inv=U) == EALIGN
    for n in ("dY", "x", "Z", "W1", "W2", "off", "dX", "dW1", "dW2"):
        assert bwd(**{n: None}) == ENULL and bwd(**{n: U}) == EALIGN, n
    assert bwd(ws=None) == EWORKSPACE and bwd(wsb=need - 1) == EWORKSPACE and bwd(ws=U) == EALIGN


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_oracle_gradients_against_differences(act):
    rng = np.random.default_rng(2)
    offsets = np.array([0, 4, 4, 9])
    X, Wg, Wu = rng.standard_normal((11, 6)), rng.standard_normal((3, 6, 10)), rng.standard_normal((3, 6, 10))
    W2, dY = rng.standard_normal((3, 10, 6)), rng.standard_normal((11, 6))
    loss = lambda X, Wg, Wu, W2: (O.glu_fwd(X, Wg, Wu, W2, act, offsets)[3] * dY).sum()
    G, Up, _, _ = O.glu_fwd(X, Wg, Wu, W2, act, offsets)
    grads = O.glu_bwd(dY, X, G, Up, Wg, Wu, W2, act, offsets)[3:]
    args = [X, Wg, Wu, W2]
    for n, g in enumerate(grads):
        d = rng.standard_normal(args[n].shape)
        h = 1e-6
        up, down = ([a + s * h * d if i == n else a for i, a in enumerate(args)] for s in (1, -1))
        assert abs((loss(*up) - loss(*down)) / (2 * h) - (g * d).sum()) < 1e-5 * max(1, abs((g * d).sum())), n
