"""What the dropless block with gated experts refuses before it launches anything."""
import pytest
import torch

from paper_2407_00599_amd.api import mx4_shapes
from paper_2407_00599_amd.layer import DroplessBlock


def test_unknown_ffn_is_refused():
    for ffn in ("silu", "relu", None, ""):
        with pytest.raises(ValueError):
            DroplessBlock(4, 64, 64, 2, 1, device="cpu", ffn=ffn)
    for ffn, act in (("gelu", None), ("swiglu", 0), ("geglu", 1)):
        assert DroplessBlock(4, 64, 64, 2, 1, ffn=ffn, device="cpu").act == act


def test_buffers_of_gated_experts():
    b = DroplessBlock(4, 64, 72, 2, 1, device="cpu", ffn="swiglu")
    assert b.Z.shape == (4, 144) and b.dW1.shape == (2, 64, 144) and not hasattr(b, "Zq")
    b = DroplessBlock(4, 64, 72, 2, 1, device="cpu", ffn="swiglu", training=False)
    assert not hasattr(b, "Z") and not hasattr(b, "dW1")


def test_four_bits_only_of_gated_experts_and_only_to_serve():
    plain, gated = (DroplessBlock(4, 64, 72, 2, 1, device="cpu", ffn=f) for f in ("gelu", "swiglu"))
    W = {"W1": torch.zeros(2, 64, 144), "W2": torch.zeros(2, 72, 64)}
    with pytest.raises(ValueError):
        plain.quantise(W)
    with pytest.raises(ValueError):
        plain.infer(torch.zeros(4, 64), {"W1q": None})
    with pytest.raises(ValueError):
        gated.forward(torch.zeros(4, 64), {"W1q": None})
    for bad in ({"W1": torch.zeros(2, 64, 72)}, {"W2": torch.zeros(2, 64, 72)}):
        with pytest.raises(ValueError):
            gated.quantise(dict(W, **bad))
    with pytest.raises(ValueError):
        gated.quantise(W)                      # tensors must live on the GPU


def test_weights_of_other_sizes():
    """refused in front of the first launch: W1 of experts with one projection, and 4 bits of another block's weights"""
    gated = DroplessBlock(4, 64, 72, 2, 1, device="cpu", ffn="swiglu")
    x = torch.zeros(4, 64)
    good = {"W1": torch.zeros(2, 64, 144), "W2": torch.zeros(2, 72, 64)}
    for bad in ({"W1": torch.zeros(2, 64, 72)}, {"W2": torch.zeros(2, 64, 72)}, {"W1": torch.zeros(1, 64, 144)}):
        for call in (gated.forward, gated.infer):
            with pytest.raises(ValueError, match="has the shape"):
                call(x, dict(good, **bad))
    bits = lambda E, M, H: {n + t: torch.zeros(shape, dtype=torch.uint8) for n, rows, cols in (("W1", M, 2 * H), ("W2", H, M))
                            for t, shape in zip("qs", mx4_shapes(E, rows, cols, True))}
    for E, M, H in ((2, 64, 64), (2, 32, 72), (1, 64, 72)):
        with pytest.raises(ValueError, match="has the shape"):
            gated.infer(x, bits(E, M, H))
    with pytest.raises((ValueError, KeyError)) as e:       # the right sizes: it is the missing norm weights or the host's tensors
        gated.infer(x, bits(2, 64, 72))
    assert "has the shape" not in str(e.value)
