"""What the dropless block refuses before it allocates anything."""
import pytest

from paper_2407_00599_amd.layer import DroplessBlock


def test_unknown_norm_or_gate_is_refused():
    for kw in ({"norm": "layernorm"}, {"norm": None}, {"gate": "row"}, {"gate": None}):
        with pytest.raises(ValueError):
            DroplessBlock(4, 64, 64, 2, 1, device="cpu", **kw)
    for norm in ("rms", "layer"):
        assert DroplessBlock(4, 64, 64, 2, 1, norm=norm, device="cpu").layer == (norm == "layer")
