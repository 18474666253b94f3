"""What the binding of the training operators does before the library is called; without a
GPU."""
import pytest
import torch

from paper_2606_10650_amd import train


def test_adamw_states_come_together():
    x = torch.zeros(8)
    for kw in (dict(m=x), dict(v=x)):
        with pytest.raises(ValueError, match="together"):
            train.AdamW().add(x, x, **kw)
