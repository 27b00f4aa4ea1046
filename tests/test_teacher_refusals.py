"""Refusals of set_teacher, on the host (no GPU)."""
import pytest
import torch

from paper_2211_12858_amd.driver import Booster


@pytest.mark.parametrize("values", ["probs", "", None, 0, ["logits"]])
def test_unknown_kind_of_values(values):
    b = Booster.__new__(Booster)  # without the device's part
    b.loss, b.n, b.d, b._F, b.teacher = "distill", 6, 4, torch.zeros((4, 6)), None
    with pytest.raises(ValueError, match="log_probs.*logits"):
        b.set_teacher(torch.zeros((2, 6), dtype=torch.int32), torch.zeros((2, 6)), values)
    assert b.teacher is None
