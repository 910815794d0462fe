"""The 8-bit form of whole tensors at once, for tests whose tensors the checker's loops over blocks take too long for
(oracle/ragged_oracle.py: store8, scale_byte).  test_eight_bits_cpu.py compares the two."""
import numpy as np

BLOCK = 32


def scale_bytes(top):
    """Scale byte of every largest magnitude in `top`."""
    top = np.asarray(top, np.float64)
    out = np.full(top.shape, 255, np.int64)
    live = np.isfinite(top)
    t = top[live]
    x = np.frexp(t)[1] - 1
    b = np.minimum(x + 127 + (t >= 127.5 * np.exp2(x - 6.0)), 254)
    out[live] = np.where(t < 2.0 ** -126, t >= 127 * 2.0 ** -133, b)
    return out


def block_tops(x):
    """Largest magnitude of every block of 32 columns; NaN and infinities as infinity."""
    rows, cols = x.shape
    a = np.zeros((rows, -(-cols // BLOCK) * BLOCK))
    a[:, :cols] = np.where(np.isfinite(x), np.abs(x), np.inf)
    return a.reshape(rows, -1, BLOCK).max(2)


def store8(x):
    """x [rows, cols] -> (q int8, scales uint8)"""
    x = np.asarray(x, np.float64)
    s = scale_bytes(block_tops(x))
    wide = np.repeat(s, BLOCK, 1)[:, :x.shape[1]]
    live = wide != 255
    q = np.zeros(x.shape, np.int8)
    q[live] = np.clip(np.rint(x[live] / np.exp2(wide[live] - 133.0)), -127, 127)
    return q, s.astype(np.uint8)


def kept_is_near(q, s, z, dz, what):
    """(q, s) is the kept form of z, which is known to +-dz: the scale of a magnitude in that range, and the nearest whole number."""
    s = s.astype(np.int64)
    lo, hi = block_tops(np.maximum(np.abs(z) - dz, 0)), block_tops(np.abs(z) + dz)
    assert ((scale_bytes(lo) <= s) & (s <= scale_bytes(hi))).all(), what
    step = np.repeat(np.exp2(s - 133.0), BLOCK, 1)[:, :z.shape[1]]
    assert (np.abs(q * step - z) <= step / 2 + dz).all(), what
