"""Float64 checker of the dropless block's operators, written from their definitions: rows that lie expert by expert, the products over
them, the 8-bit form of a tensor, the expert FFN whose backward pass reads that form, and the norms around the block.  It shares no code
with the HIP path."""
import numpy as np
from scipy.special import erf

BLOCK = 32


def plan(idx, slot, counts, C):
    """offsets [E + 1], row [S, k] (-1: none), row_inv [S k]: the rows one by one, expert by expert."""
    S, k = idx.shape
    E = len(counts)
    offsets = np.zeros(E + 1, np.int64)
    for e in range(E):
        offsets[e + 1] = offsets[e] + min(int(counts[e]), C)
    row = np.full((S, k), -1, np.int64)
    inv = np.full(S * k, -1, np.int64)
    for t in range(S):
        for j in range(k):
            if slot[t, j] >= 0:
                row[t, j] = offsets[idx[t, j]] + slot[t, j]
                inv[row[t, j]] = t * k + j
    return offsets, row, inv


def scale_byte(top):
    """Scale byte for a block's largest magnitude, step = 2^(byte - 133)."""
    if not np.isfinite(top):
        return 255
    if top < 2.0 ** -126:                                    # the smallest step, and where the next one takes over
        return int(top >= 127 * 2.0 ** -133)
    x = int(np.frexp(top)[1]) - 1
    return min(x + 127 + int(top >= 127.5 * 2.0 ** (x - 6)), 254)


def store8(x):
    """x [rows, cols] -> (q int8, scales uint8)"""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    q, s = np.zeros((rows, cols), np.int8), np.zeros((rows, nb), np.uint8)
    for r in range(rows):
        for n in range(nb):
            v = x[r, n * BLOCK:(n + 1) * BLOCK]
            finite = np.isfinite(v).all()
            s[r, n] = scale_byte(np.abs(v).max() if finite else np.inf)
            if finite:
                q[r, n * BLOCK:(n + 1) * BLOCK] = np.clip(np.rint(v / 2.0 ** (int(s[r, n]) - 133)), -127, 127)
    return q, s


def load8(q, s):
    step = np.where(s == 255, np.nan, np.exp2(s.astype(np.float64) - 133))
    return q.astype(np.float64) * np.repeat(step, BLOCK, axis=1)[:, :q.shape[1]]


def gelu(z):
    return z * 0.5 * (1 + erf(z / np.sqrt(2)))


def gelu_grad(z):
    return 0.5 * (1 + erf(z / np.sqrt(2))) + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)


def rows_of(x, inv, k):
    out = np.zeros((len(inv), x.shape[1]))
    live = inv >= 0
    out[live] = x[inv[live] // k]
    return out


def gemm(X, W, offsets):
    """X W[e] for the rows of expert e, zeros behind them; W [E, K, N]"""
    Y = np.zeros((X.shape[0], W.shape[2]))
    for e in range(len(W)):
        Y[offsets[e]:offsets[e + 1]] = X[offsets[e]:offsets[e + 1]] @ W[e]
    return Y


def wgrad(X, dY, offsets):
    return np.stack([X[a:b].T @ dY[a:b] for a, b in zip(offsets[:-1], offsets[1:])])


def ffn_bwd(dY, X, z, W1, W2, offsets):
    """dX, dW1, dW2 of Y = GeLU(Z) W2, Z = X W1, at the kept pre-activation z"""
    dZ = gemm(dY, W2.transpose(0, 2, 1), offsets) * gelu_grad(z)
    return gemm(dZ, W1.transpose(0, 2, 1), offsets), wgrad(X, dZ, offsets), wgrad(gelu(z), dY, offsets)


def norm(v, w, b, eps, layer):
    """n(v), mean [S], rstd [S], normalised value"""
    mean = v.mean(1) if layer else np.zeros(len(v))
    d = v - mean[:, None]
    rstd = 1 / np.sqrt((d * d).mean(1) + eps)
    hat = d * rstd[:, None]
    return hat * w + (0 if b is None else b), mean, rstd, hat


def norm_grad(up, hat, rstd, w, layer):
    """gradients of v, w and b for the upstream gradient of n(v)"""
    g = up * w
    dv = g - hat * (g * hat).mean(1, keepdims=True)
    if layer:
        dv = dv - g.mean(1, keepdims=True)
    return dv * rstd[:, None], (up * hat).sum(0), up.sum(0)


def spread_gate(gate, kind):
    return np.ones((1, 1)) if kind == "none" else gate[:, None] if kind == "token" else gate[None, :]


def norm_residual(h, x, w, b, gate, kind, alpha, eps, layer):
    n, mean, rstd, hat = norm(h, w, b, eps, layer)
    return x + alpha * spread_gate(gate, kind) * n, mean, rstd, hat, n


def norm_residual_grad(dy, n, hat, rstd, w, gate, kind, alpha, layer):
    dh, dw, db = norm_grad(alpha * spread_gate(gate, kind) * dy, hat, rstd, w, layer)
    dgate = None if kind == "none" else (alpha * dy * n).sum(1 if kind == "token" else 0)
    return dh, dw, db, dgate
