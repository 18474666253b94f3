"""The norm at the ends of float32's range, and at the largest numbers of rows, against its
formula in float64.  Tolerances are those of the same outputs at ordinary values.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

LEAST = 448 * 2.0 ** -126     # of a row's largest value, where 8 bits begin


def _train():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import train
    return train


def formula(x, w, eps):
    x = x.double()
    return x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()


@pytest.mark.parametrize("D", [1, 64, 777, 4096])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_fp8_small_rows(D, dtype):
    """Rows whose largest values go down to the smallest numbers, with zeros among them:
    codes are finite and within their rounding, or zero below the least value."""
    tr = _train()
    gen = torch.Generator(device="cuda").manual_seed(D)
    tops = torch.tensor([2.0 ** -e for e in range(60, 134)] + [0.0], device="cuda", dtype=torch.float64)
    x = 2 * torch.rand((len(tops), D), generator=gen, device="cuda", dtype=torch.float64) - 1
    x[:, ::3] = 0
    x[:, 0] = 1
    x = (x * tops[:, None]).to(dtype)
    w = torch.ones(D, device="cuda", dtype=dtype)
    y, _, scale = tr.rms_norm_fp8(x, w, eps=4.0)        # y = x / 2
    torch.cuda.synchronize()
    want = formula(x, w, 4.0)
    top = want.abs().amax(-1)
    assert torch.isfinite(y.float()).all() and torch.isfinite(scale).all()
    none = top < LEAST
    assert none.any() and not none.all()
    assert not y[none].float().any() and not scale[none].any()
    y, scale, want, top = (t[~none].double() for t in (y, scale, want, top))
    assert ((scale - top / 448).abs() <= 1e-5 * top / 448).all()
    # half a spacing: 2^-4 of a value, 2^-10 of the scale below the least normal code
    assert ((y * scale[:, None] - want).abs() <= want.abs() * (2.0 ** -4 + 1e-5) + scale[:, None] * 2.0 ** -10).all()
    assert (y.abs().amax(-1) == 448).all()
