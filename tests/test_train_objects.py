"""QkRotation and PackedAttention marshal their tensors and settings when they are made: none of them can be exchanged afterwards, so that
all calls of an object, in either direction and whatever way they take through the binding, mean the same ones (no GPU needed)."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("name,attributes", [
    ("QkRotation", ("inv_freq", "D", "q_weight", "k_weight", "eps", "layout", "workspace")),
    ("PackedAttention", ("seq_offsets", "group_offsets", "causal", "sm_scale", "status_dev", "workspace", "out", "lse", "dq", "dk", "dv")),
])
def test_what_was_marshalled_is_not_exchanged(name, attributes):
    from paper_2605_07114_b200 import hora
    op = object.__new__(getattr(hora, name))
    for x in attributes:
        with pytest.raises(AttributeError):
            setattr(op, x, torch.zeros(4))
