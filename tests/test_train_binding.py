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


def test_workspace_is_memory_of_its_size():
    """Another device's memory, and a tensor that repeats a few bytes or skips some, are
    refused: the library would write past them."""
    cpu = torch.device("cpu")
    byte = torch.zeros(512, dtype=torch.uint8)
    for bad in (byte[:1].expand(1 << 20), byte[::2], torch.empty(512, dtype=torch.uint8, device="meta")):
        with pytest.raises(ValueError, match="workspace"):
            train._space(bad, 100, cpu)
    assert train._space(byte, 512, cpu)[0] is byte and train._space(byte.view(torch.int32), 512, cpu)[1] == 512
    assert train._space(byte, 513, cpu)[1] == 513 and train._space(None, 0, cpu)[1] == 256
