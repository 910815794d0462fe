"""What the dropless block with gated experts refuses before it launches anything."""
import pytest
import torch

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
