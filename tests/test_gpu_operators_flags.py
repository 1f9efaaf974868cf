"""Flags without a truth value raise what they raise, before anything is launched."""
import pytest
import torch


@pytest.mark.gpu
def test_flags_without_a_truth_value():
    from paper_2607_19378_b200 import hyenand as hn
    x, two = torch.zeros((2, 3, 8), device="cuda"), torch.zeros(2)
    with pytest.raises(RuntimeError, match="ambiguous"):
        hn.Recurrence(8, 2, 3).forward(x, x, x, x, marks=two)
    with pytest.raises(RuntimeError, match="ambiguous"):
        hn.Block((8,), 2, 3).forward(x, x, stats=two)
    assert len(hn.Recurrence(8, 2, 3).forward(x, x, x, x, marks=torch.ones(1))) == 3 and len(hn.Block((8,), 2, 3).forward(x, x, stats=0)) == 2
