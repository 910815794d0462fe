"""GPU parity of the gated FFN served from 4 bits with either of its products in tiles of 256 x 256, rows as they lie and through the map.  The test, its
oracle and its bounds are those of test_gpu_mx4.py."""
import pytest

import test_gpu_mx4 as base
from test_mx4_choice_cpu import tile

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,act", [("f32", "silu"), ("bf16", "silu"), ("bf16", "gelu")])
@pytest.mark.parametrize("ns,behind,M,H,gather,tiles", [((600, 0, 830), 0, 520, 3592, False, (256, 128)), ((600, 0, 830), 5, 520, 2568, True, (256, 128)),
                                                        ((1300, 257), 3, 8200, 72, True, (128, 256))])
def test_glu(ns, behind, M, H, gather, tiles, dtype, act):
    R, E = sum(ns) + behind, len(ns)
    assert (tile(R, E, 2 * H, M), tile(R, E, M, H)) == tiles
    base.test_glu(ns, behind, M, H, gather, dtype, act)
