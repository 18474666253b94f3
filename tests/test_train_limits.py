"""The largest sizes that the training operators take, without a GPU: what no launch can hold
is refused before anything is enqueued."""
import ctypes

import pytest
import torch

from paper_2606_10650_amd import dla, train

FAKE = 0x10000


@pytest.mark.parametrize("states", [dla.DLA_F32, train.DLA_STATE_FP8])
def test_adamw_elements(states):
    def step(n):
        t = train.AdamWTensor(FAKE, None, FAKE, FAKE, FAKE, FAKE, FAKE, n, 0.0)
        p = train.AdamWParams(1e-3, 0.9, 0.99, 1e-8, 1, 0, 0, states, 0, None)
        return train.lib().dla_adamw_step(ctypes.byref(t), 1, ctypes.byref(p), None)

    for n in ((1 << 36) - 4095, 1 << 36, 1 << 40):
        assert step(n) == dla.DLA_ERR_UNSUPPORTED
    assert step((1 << 40) + 1) == dla.DLA_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_heads(dtype):
    """65535 of them, in a forward call of up to 6 tokens 2^21 - 1."""
    n = ctypes.c_size_t(0)

    def ask(heads, T, backward=False):
        d = train._desc(1, heads, heads, T, 64, 64, dtype)
        return train.lib().dla_recurrence_workspace_size(d, int(backward), ctypes.byref(n))

    for T in (0, 1, 6):
        assert ask((1 << 21) - 1, T) == dla.DLA_OK and n.value == 0
        assert ask(1 << 21, T) == dla.DLA_ERR_UNSUPPORTED
        assert ask(65535, T, True) == dla.DLA_OK
        assert ask(65536, T, True) == dla.DLA_ERR_UNSUPPORTED
    assert ask(65535, 7) == dla.DLA_OK and ask(65536, 7) == dla.DLA_ERR_UNSUPPORTED
    assert ask(1, 1 << 30) == dla.DLA_OK and ask(1, (1 << 30) + 1) == dla.DLA_ERR_UNSUPPORTED
