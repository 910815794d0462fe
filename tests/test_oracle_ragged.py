"""Pins of the checker of the dropless block's operators: the plan against a queue simulation, the 8-bit form by its defining
properties, gradients against central differences."""
import numpy as np
import pytest

from oracle import moe_oracle as MO
from oracle import ragged_oracle as O


@pytest.mark.parametrize("S,E,k,C", [(1, 1, 1, 1), (7, 3, 2, 2), (40, 8, 3, 40), (33, 5, 5, 9)])
def test_plan_is_the_experts_queues_one_after_the_other(S, E, k, C):
    rng = np.random.default_rng(S)
    idx = np.stack([rng.permutation(E)[:k] for _ in range(S)]).astype(np.int32)
    queues = [[] for _ in range(E)]
    slot = np.full((S, k), -1, np.int32)
    for j in range(k):
        for t in range(S):
            q = queues[idx[t, j]]
            if len(q) < C:
                slot[t, j] = len(q)
            q.append(t * k + j)
    counts = np.array([len(q) for q in queues])
    offsets, row, inv = O.plan(idx, slot, counts, C)
    flat = [c for q in queues for c in q[:C]]
    assert list(inv[:len(flat)]) == flat and (inv[len(flat):] == -1).all() and offsets[-1] == len(flat)
    for t in range(S):
        for j in range(k):
            assert row[t, j] == (-1 if slot[t, j] < 0 else flat.index(t * k + j))


def test_eight_bit_form():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 100)) * np.exp2(rng.integers(-40, 40, (50, 1)))
    x[3] = 0
    q, s = O.store8(x)
    back = O.load8(q, s)
    step = np.repeat(np.exp2(s.astype(float) - 133), 32, 1)[:, :100]
    assert (np.abs(back - x) <= step / 2).all() and (back[3] == 0).all()
    top = np.abs(x[:, :32]).max(1)
    k = np.abs(q[:, :32].astype(int)).max(1)
    assert ((k >= 64) & (k <= 127))[top > 0].all()                      # the largest magnitude uses the upper half of the range
    assert (O.store8(back)[0] == q).all() and (O.load8(*O.store8(back)) == back).all()      # what is kept is kept exactly
    # the doubled step starts where a / step would round to 128
    for a, b in ((127.49, 133), (127.5, 134), (64, 133), (63.99, 133), (63.7, 132), (1.0, 127)):
        assert O.scale_byte(a) == b, a
    assert O.scale_byte(np.inf) == 255 and O.scale_byte(3.4e38) == 254 and O.scale_byte(1e-40) == 0
    assert np.isnan(O.load8(*O.store8(np.array([[1.0, np.nan] + [0.0] * 38])))[0, :32]).all()


def test_ffn_gradients_against_differences():
    """Small whole numbers make every pre-activation a kept value, so the kept form is the pre-activation itself."""
    rng = np.random.default_rng(2)
    offsets = np.array([0, 4, 4, 9])
    X, W1 = rng.integers(-1, 2, (11, 6)) / 4, rng.integers(-1, 2, (3, 6, 40)) / 4
    W2, dY = rng.standard_normal((3, 40, 6)), rng.standard_normal((11, 6))
    loss = lambda X, W1, W2: (O.gemm(O.gelu(O.gemm(X, W1, offsets)), W2, offsets) * dY).sum()
    z = O.load8(*O.store8(O.gemm(X, W1, offsets)))
    assert (z == O.gemm(X, W1, offsets)).all()
    grads = O.ffn_bwd(dY, X, z, W1, W2, offsets)
    for n, g in enumerate(grads):
        for _ in range(12):
            args = [X.copy(), W1.copy(), W2.copy()]
            at = tuple(rng.integers(0, d) for d in g.shape)
            args[n][at] += 1e-5
            up = loss(*args)
            args[n][at] -= 2e-5
            assert abs((up - loss(*args)) / 2e-5 - g[at]) < 1e-7 * (1 + abs(g[at])), (n, at)


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("kind", ["none", "channel", "token"])
def test_norm_gradients_against_differences(layer, kind):
    rng = np.random.default_rng(3)
    S, M, alpha, eps = 5, 16, 0.7, 1e-5
    h, x, dy, w = rng.standard_normal((S, M)) + 0.3, rng.standard_normal((S, M)), rng.standard_normal((S, M)), rng.standard_normal(M)
    b = rng.standard_normal(M) if layer else None
    gate = None if kind == "none" else rng.random(S if kind == "token" else M)
    names = {"h": h, "w": w, **({"b": b} if layer else {}), **({"gate": gate} if gate is not None else {})}

    def loss(**kw):
        a = dict(names, **kw)
        return (O.norm_residual(a["h"], x, a["w"], a.get("b"), a.get("gate"), kind, alpha, eps, layer)[0] * dy).sum()
    _, _, rstd, hat, n = O.norm_residual(h, x, w, b, gate, kind, alpha, eps, layer)
    dh, dw, db, dgate = O.norm_residual_grad(dy, n, hat, rstd, w, gate, kind, alpha, layer)
    for name, g in (("h", dh), ("w", dw), ("b", db), ("gate", dgate)):
        if name not in names:
            continue
        for at in np.ndindex(*g.shape):
            v = names[name].copy()
            v[at] += 1e-5
            up = loss(**{name: v})
            v[at] -= 2e-5
            assert abs((up - loss(**{name: v})) / 2e-5 - g[at]) < 1e-7 * (1 + abs(g[at])), (name, at)


def test_dropless_equals_the_padded_layer():
    """With room for every choice, rows without padding carry what the capacity-padded layer computes."""
    rng = np.random.default_rng(4)
    S, M, H, E, k = 24, 8, 16, 4, 2
    x, Wg = rng.standard_normal((S, M)), rng.standard_normal((M, E)).astype(np.float32)
    W1, W2 = rng.standard_normal((E, M, H)), rng.standard_normal((E, H, M))
    r = MO.layer_fwd(x, Wg, None, W1, W2, k, E / k, True)
    offsets, row, inv = O.plan(r["idx"], r["slot"], r["counts"], S)
    Y = O.gemm(O.gelu(O.gemm(O.rows_of(x, inv, k), W1, offsets)), W2, offsets)
    y = (np.asarray(r["w"], np.float64)[:, :, None] * Y[row]).sum(1)
    np.testing.assert_allclose(y, r["y"], rtol=1e-10, atol=1e-12)
