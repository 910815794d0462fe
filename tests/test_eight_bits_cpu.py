"""The whole-tensor 8-bit form of the tests is the checker's."""
import numpy as np

import eight_bits
from oracle import ragged_oracle as O


def test_whole_tensors_like_blocks():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((60, 104)) * np.exp2(rng.integers(-140, 127, (60, 104)) * (rng.random((60, 104)) < 0.2))
    x[0] = 0
    x[1, 3], x[2, 40], x[3, 100] = np.inf, np.nan, -np.inf
    for r, top in enumerate((127.0, 127.49, 127.5, 255.0, 3.4028234663852886e38, 2.0 ** -126, 0.996 * 2.0 ** -126, 2.0 ** -127, 1e-45), 4):
        x[r] = 0
        x[r, 7], x[r, 50] = top, -top
    q, s = O.store8(x)
    q2, s2 = eight_bits.store8(x)
    assert np.array_equal(q, q2) and np.array_equal(s, s2)
