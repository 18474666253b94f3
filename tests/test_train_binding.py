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


def test_calls_go_to_the_tensors_device(monkeypatch):
    """Kernels are launched on the current device: a call on another device's tensors makes
    that one current, and has its stream."""
    current, seen = [0], []

    class Device:
        def __init__(self, device):
            self.index = device.index

        def __enter__(self):
            self.was, current[0] = current[0], self.index

        def __exit__(self, *_):
            current[0] = self.was

    class Lib:
        def dla_call(self, *args):
            seen.append((current[0], *args))
            return 0

    monkeypatch.setattr(train, "_current_device", lambda: current[0])
    monkeypatch.setattr(train, "_stream", lambda device: f"stream {device.index} of {current[0]}")
    monkeypatch.setattr(train, "lib", Lib)
    monkeypatch.setattr(torch.cuda, "device", Device)
    for i in (0, 1):
        train._run("dla_call", torch.device("cuda", i), 5)
    assert seen == [(0, 5, "stream 0 of 0"), (1, 5, "stream 1 of 1")] and current == [0]
