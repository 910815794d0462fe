"""The vectorised 4-bit form of the tests is the oracle's."""
import numpy as np

import four_bits as F
from oracle import mx4_oracle as O


def test_it_is_the_oracles():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((60, 136)) * np.exp2(rng.integers(-130, 126, (60, 1)))
    x[::5] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.0, -0.0, -0.25, -7.0, -5.0], (12, 136))
    x[1], x[2, 5], x[3, 70], x[4] = 0, np.inf, np.nan, 3.4e38 * (rng.random(136) - 0.5)
    x = x.astype(np.float32).astype(np.float64)
    (q, s), (rq, rs) = F.store(x), O.store(x)
    assert np.array_equal(q, rq) and np.array_equal(s, rs)
    assert np.array_equal(F.kept(x), O.kept(x), equal_nan=True)
    y = rng.standard_normal((30, 100))
    for d in (0 * y, 1e-3 * np.abs(y), np.full_like(y, 0.05)):
        for got, ref in zip(F.kept_range(y, d), O.kept_range(y, d)):
            assert np.array_equal(got, ref)
