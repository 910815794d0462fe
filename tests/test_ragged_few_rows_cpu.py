"""Which forward calls the kernels for few rows take, seen from the workspace that they and, in bf16, nothing else of a forward call ask for."""
from paper_2407_00599_amd import api


def few(R, E, M=1024, H=4096, dtype=api.MOE_BF16):
    return api.moe_ragged_ffn_workspace_bytes(dtype, R, E, M, H, 1, 0) > 0


def test_bounded_whatever_the_number_of_experts():
    """They read an expert's weights again for every 16 rows of it, and all rows may be one expert's: 64 rows at most, 32 of few experts."""
    for E in (1, 4, 8, 64, 256):
        assert few(1, E) and few(32, E)
        assert few(64, E) == (E >= 8)
        for R in (65, 128, 512, 2048):
            assert not few(R, E), (R, E)
    assert not few(8, 8, 1024, 1024) and not few(8, 8, 256, 1024)
