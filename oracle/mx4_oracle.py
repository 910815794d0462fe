"""Float64 oracle of microscaled 4-bit floating point and of the products from it, written from their definitions; it shares no code with the
HIP path."""
import numpy as np

from oracle import ragged_oracle as R

BLOCK, CHUNK = 32, 512
SIZES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def scale_byte(top):
    """of a block's largest magnitude; 2^(byte - 127)"""
    if not np.isfinite(top):
        return 255
    if top == 0:
        return 0
    x = int(np.frexp(top)[1]) - 1
    return min(max(x - 2 + 127 + int(top / 2.0 ** (x - 2) >= 7), 0), 252)       # 6 2^125 is a number, 8 2^125 is not


def code(v, b):
    """of values with scale byte b: the nearest size, of two the even one"""
    m = np.abs(np.asarray(v, np.float64)) / 2.0 ** (b - 127.0)
    d = np.abs(np.minimum(m, 6)[..., None] - SIZES)
    nearest = d == d.min(-1, keepdims=True)
    return np.where(nearest, np.arange(8) % 2, 2).argmin(-1) + 8 * np.signbit(v)


def store(x):
    """x [n, K] -> codes [n, blocks, 32], scale bytes [n, blocks]"""
    x = np.asarray(x, np.float64)
    n, K = x.shape
    blocks = -(-K // BLOCK)
    v = np.zeros((n, blocks * BLOCK))
    v[:, :K] = x
    v = v.reshape(n, blocks, BLOCK)
    s = np.zeros((n, blocks), np.int64)
    q = np.zeros(v.shape, np.int64)
    for r in range(n):
        for b in range(blocks):
            s[r, b] = scale_byte(np.abs(v[r, b]).max() if np.isfinite(v[r, b]).all() else np.inf)
            if s[r, b] != 255:
                q[r, b] = code(v[r, b], s[r, b])
    return q, s


def values(q, s):
    """[n, blocks * 32]"""
    step = np.where(s == 255, np.nan, 2.0 ** (s - 127.0))[..., None]
    return (np.where(q >= 8, -1, 1) * SIZES[q % 8] * step).reshape(len(q), -1)


def kept(x):
    """what 4 bits keep of x [n, K]"""
    return values(*store(x))[:, :np.shape(x)[1]]


def pack(q, s):
    """the bytes as they are held: [n, blocks * 16], [chunks, 4, n, 4]"""
    n, blocks, _ = q.shape
    b = (q[:, :, 0::2] | q[:, :, 1::2] << 4).astype(np.uint8).reshape(n, blocks * 16)
    chunks = -(-blocks // 16)
    out = np.zeros((chunks, 4, n, 4), np.uint8)
    for k in range(blocks):
        out[k // 16, k % 4, :, k % 16 // 4] = s[:, k]
    return b, out


def kept_range(x, d):
    """the least and the largest that 4 bits may keep of values known to +- d: of either scale that the largest magnitude allows"""
    lo, hi = np.zeros_like(x), np.zeros_like(x)
    for r in range(len(x)):
        for c in range(0, x.shape[1], BLOCK):
            v, e = x[r, c:c + BLOCK], d[r, c:c + BLOCK]
            scales = {scale_byte(max((np.abs(v) - e).max(), 0.0)), scale_byte((np.abs(v) + e).max())}
            at = lambda u, b: values(code(u, b)[None, None], np.array([[b]]))[0]
            lo[r, c:c + BLOCK] = np.min([at(v - e, b) for b in scales], 0)
            hi[r, c:c + BLOCK] = np.max([at(v + e, b) for b in scales], 0)
    return lo, hi


def glu(X, Wg, Wu, act, offsets):
    """A of rows X and the two halves of W1, all of them what 4 bits keep"""
    return R.gate_act(act, R.gemm(X, Wg, offsets))[0] * R.gemm(X, Wu, offsets)
