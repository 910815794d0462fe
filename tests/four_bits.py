"""The oracle's microscaled 4-bit form of whole tensors at once, for the sizes at which its loops over blocks take too long; test_four_bits_cpu.py holds it
against them."""
import numpy as np

from oracle.mx4_oracle import SIZES

MIDDLES = (SIZES[1:] + SIZES[:-1]) / 2
# what a value in the middle of two sizes is kept as: the one with the even code
EVEN = np.array([0, 2, 2, 4, 4, 6, 6])


def scale_bytes(top):
    """of blocks' largest magnitudes"""
    m, e = np.frexp(np.where(np.isfinite(top), top, 1.0))
    b = np.where(top > 0, np.clip(e + 124 + (m >= 0.875), 0, 252), 0)
    return np.where(np.isfinite(top), b, 255).astype(np.int64)


def codes(v, b):
    """codes of values whose blocks have scale bytes b (broadcast)"""
    m = np.minimum(np.abs(v) / np.exp2(b - 127.0), 6)
    below = np.searchsorted(MIDDLES, m, side="left")          # m <= MIDDLES[below]
    at = np.minimum(below, len(MIDDLES) - 1)
    return np.where((below < len(MIDDLES)) & (m == MIDDLES[at]), EVEN[at], below) + 8 * np.signbit(v)


def blocks_of(x):
    x = np.asarray(x, np.float64)
    return np.pad(x, ((0, 0), (0, -x.shape[1] % 32))).reshape(len(x), -1, 32)


def store(x):
    v = blocks_of(x)
    finite = np.isfinite(v).all(-1)
    s = scale_bytes(np.where(finite, np.abs(np.where(np.isfinite(v), v, 0)).max(-1), np.inf))
    return np.where(finite[..., None], codes(np.where(finite[..., None], v, 0), s[..., None]), 0), s


def values(q, s):
    step = np.where(s == 255, np.nan, np.exp2(s - 127.0))[..., None]
    return np.where(q >= 8, -1, 1) * SIZES[q % 8] * step


def kept(x):
    return values(*store(x)).reshape(len(x), -1)[:, :np.shape(x)[1]]


def kept_range(x, d):
    """the least and the largest that 4 bits may keep of values known to +- d"""
    v, e = blocks_of(x), blocks_of(d)
    low, high = scale_bytes(np.maximum((np.abs(v) - e).max(-1), 0)), scale_bytes((np.abs(v) + e).max(-1))
    # (a bound that a binade's border or two lie in leaves three scales at most: those in between are tried too)
    lo = hi = None
    for s in (low, high, np.minimum(low + 1, high)):
        a, b = values(codes(v - e, s[..., None]), s), values(codes(v + e, s[..., None]), s)
        lo, hi = (a, b) if lo is None else (np.minimum(lo, a), np.maximum(hi, b))
    cut = lambda t: t.reshape(len(x), -1)[:, :np.shape(x)[1]]
    return cut(lo), cut(hi)
