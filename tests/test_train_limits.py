"""The largest sizes that the training operators take, without a GPU: what no launch can hold
is refused before anything is enqueued."""
import ctypes

import pytest

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
