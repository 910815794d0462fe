"""GPU: the kept form of fp32 pre-activations next to the border between two steps.  The sums are exact in fp64 and round onto the border in
fp32, so scale and values tell which of the two the form was made from; both are compared bit for bit."""
import numpy as np
import pytest
import torch

import eight_bits
from paper_2407_00599_amd import api
from util import DEV

pytestmark = pytest.mark.gpu


# one tile of 32 x 32, and so many that they are 64 x 64
@pytest.mark.parametrize("R,H", [(40, 72), (800, 4104)])
def test_scale_of_a_sum_just_below_the_border(R, H):
    M, off = 64, 2.0 ** -30
    rng = np.random.default_rng(1)
    x = np.zeros((R, M), np.float32)
    x[:, 0] = np.exp2(rng.integers(-3, 4, R))                   # Z = x[:, 0] (W1[0] + 2^-30 W1[1]): exact in fp64
    x[:, 1] = x[:, 0] * off
    steps = rng.integers(-100, 101, H).astype(np.float64)       # odd ones among them, which a doubled step does not hold
    tie = np.zeros(H)
    blocks = (H + 31) // 32
    for b in range(blocks):
        n = 32 * b + 5                                          # the block's largest magnitude
        steps[n] = (127.5, -127.5, 127.0, -128.0)[b % 4]
        tie[n] = -np.sign(steps[n]) * (1, 1, 0, 1)[b % 4]       # below it in magnitude
    W1 = np.zeros((1, M, H), np.float32)
    W1[0, 0], W1[0, 1] = steps / 64, tie
    z = x.astype(np.float64) @ W1[0].astype(np.float64)
    on = np.arange(5, H, 32)[: 2 if blocks > 1 else 1]
    assert (np.abs(z.astype(np.float32).astype(np.float64)[:, on]) > np.abs(z[:, on])).all()
    d = lambda a: torch.from_numpy(a).to(DEV)
    Zq = torch.full((R, H), 99, dtype=torch.int8, device=DEV)
    Zs = torch.full((R, blocks), 99, dtype=torch.uint8, device=DEV)
    A, Y = torch.empty(R, H, device=DEV), torch.empty(R, M, device=DEV)
    ws = torch.empty(max(api.moe_ragged_ffn_workspace_bytes(api.MOE_F32, R, 1, M, H, 1, 0), 16), dtype=torch.uint8, device=DEV)
    offsets = torch.tensor([0, R], dtype=torch.int32, device=DEV)
    api.moe_ragged_ffn_fwd(d(x), 0, None, 1, d(W1), torch.zeros(1, H, M, device=DEV), offsets, R, 1, M, H, 0, 1, Zq, Zs, A, Y, ws)
    q, s = eight_bits.store8(z)
    assert np.array_equal(Zs.cpu().numpy(), s)
    assert np.array_equal(Zq.cpu().numpy(), q)


def test_sums_beyond_fp32_are_infinities():
    """What fp32 cannot hold is kept as NaN blocks, like an infinity; the largest values that it holds saturate."""
    M, H = 8, 64
    x = torch.zeros(3, M, device=DEV)
    x[0, 0], x[1, 0], x[2, 0] = 2.0 ** 100, 2.0 ** 100, 1.0
    W1 = torch.zeros(1, M, H, device=DEV)
    W1[0, 0, 3], W1[0, 0, 40] = 2.0 ** 30, (1 - 2.0 ** -12) * 2.0 ** 28
    Zq, Zs = torch.empty(3, H, dtype=torch.int8, device=DEV), torch.empty(3, 2, dtype=torch.uint8, device=DEV)
    A, Y = torch.empty(3, H, device=DEV), torch.empty(3, M, device=DEV)
    api.moe_ragged_ffn_fwd(x, 0, None, 1, W1, torch.zeros(1, H, M, device=DEV), torch.tensor([0, 3], dtype=torch.int32, device=DEV), 3, 1, M, H,
                           0, 1, Zq, Zs, A, Y, None)
    assert Zs.cpu().tolist() == [[255, 254], [255, 254], [157, 155]]
    assert int(Zq[0, 40]) == 127 and int(Zq[2, 3]) == 64 and int(Zq[2, 40]) == 64
