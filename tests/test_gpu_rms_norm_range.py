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


@pytest.mark.parametrize("D", [1, 64, 777, 2048, 16384])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_rows_whose_squares_leave_the_range(D, dtype, eps):
    """Rows of 2^-124 to 2^126, whose squares reach neither end of float32: y and r as for
    ordinary rows, and a gradient too."""
    tr = _train()
    gen = torch.Generator(device="cuda").manual_seed(D)
    size = torch.tensor([2.0 ** e for e in range(-124, 127, 5)], device="cuda", dtype=torch.float64)
    x = torch.rand((len(size), D), generator=gen, device="cuda", dtype=torch.float64) + 0.5
    x[:, 1::2] *= -1
    x = (x * size[:, None]).to(dtype)
    w = (1 + 0.2 * torch.randn(D, generator=gen, device="cuda")).to(dtype)
    y, _, rstd = tr.rms_norm(x, w, eps=eps)
    codes, _, scale = tr.rms_norm_fp8(x, w, eps=eps)
    torch.cuda.synchronize()
    want = formula(x, w, eps)
    r = 1 / (x.double().square().mean(-1) + eps).sqrt()
    # r of the largest rows is below the normal numbers: three bits fewer
    assert ((rstd.double() - r).abs() <= r * 1e-5 + 2.0 ** -149).all()
    tol = (2.0 ** -8 if dtype == torch.bfloat16 else 0) + 1e-5
    # y is float32's own spacing off where it is below the normal numbers
    assert ((y.double() - want).abs() <= tol * want.abs() + 2.0 ** -(133 if dtype == torch.bfloat16 else 149)).all()
    some = want.abs().amax(-1) > LEAST
    got = codes.double() * scale.double()[:, None]
    assert ((got - want).abs() <= want.abs() * (2.0 ** -4 + 1e-5) + scale.double()[:, None] * 2.0 ** -10)[some].all()
    if eps == 0:
        dx, dw = tr.rms_norm_backward(y, x, w, rstd)
        fit = size < 2.0 ** 120     # dx is of dy r's size: normal there
        n, dn = want / w.double(), y.double() * w.double()
        dx64 = (dn - n * (dn * n).mean(-1, keepdim=True)) * r[:, None]
        off = (dx.double() - dx64).norm(dim=-1) / (dn * r[:, None]).norm(dim=-1)
        assert (off[fit] <= tol).all() and torch.isfinite(dw).all()


@pytest.mark.parametrize("D", [64, 777, 2048])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_zeros_without_eps(D, dtype):
    """eps = 0 and nothing to divide by: r, y, codes and scale are zero, and the gradient is
    what reaches h itself."""
    tr = _train()
    x = torch.ones((3, D), device="cuda", dtype=dtype)
    x[1] = 0
    w = torch.ones(D, device="cuda", dtype=dtype)
    y, _, rstd = tr.rms_norm(x, w, eps=0.0)
    codes, _, scale = tr.rms_norm_fp8(x, w, eps=0.0)
    dx, dw = tr.rms_norm_backward(torch.ones_like(x), x, w, rstd, dres=3 * torch.ones_like(x))
    torch.cuda.synchronize()
    assert rstd.tolist() == [1, 0, 1] and not y[1].any() and (y[::2] == 1).all()
    assert not codes[1].float().any() and scale[1] == 0 and (codes[::2].float() == 448).all()
    assert (dx[1] == 3).all() and (dw == 2).all()


def test_more_rows_than_a_launch_takes():
    """2^26 + 3 short rows, one wave each: more than 2^32 threads."""
    tr = _train()
    N, D = 2 ** 26 + 3, 2
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((N, D), generator=gen, device="cuda", dtype=torch.bfloat16)
    r = torch.randn((N, D), generator=gen, device="cuda", dtype=torch.bfloat16)
    w = torch.tensor([1.0, -2.0], device="cuda", dtype=torch.bfloat16)
    H = x.float() + r.float()
    R = 1 / (H.square().mean(-1) + 1e-6).sqrt()
    y, h, rstd = tr.rms_norm(x, w, r)
    assert torch.equal(h, H.bfloat16())
    assert ((rstd - R).abs() <= 1e-5 * R).all()
    want = H * R[:, None] * w.float()
    assert ((y.float() - want).abs() <= (2.0 ** -8 + 1e-5) * want.abs()).all()
    del rstd, y, h
    codes, h, scale = tr.rms_norm_fp8(x, w, r)
    assert torch.equal(h, H.bfloat16())
    top = want.abs().amax(-1)
    assert ((scale - top / 448).abs() <= 1e-5 * top / 448).all()
    off = (codes.float() * scale[:, None] - want).abs()
    assert (off <= want.abs() * (2.0 ** -4 + 1e-5) + scale[:, None] * 2.0 ** -10).all()
    dx, dw = tr.rms_norm_backward(y := want.bfloat16(), h, w, R)
    torch.cuda.synchronize()
    n, dn = h.float() * R[:, None], y.float() * w.float()
    want = (dn - n * (dn * n).mean(-1, keepdim=True)) * R[:, None]
    assert ((dx.float() - want).abs() <= (2.0 ** -8 + 1e-5) * (dn.abs().amax(-1) * R)[:, None] * 2).all()


def test_broadcast_rows_are_refused():
    """One row for all is no rows apart: rms_norm takes none (the RMSNorm function copies)."""
    tr = _train()
    from paper_2606_10650_amd import dla
    x, w = torch.ones((1, 64), device="cuda"), torch.ones(64, device="cuda")
    for call in (tr.rms_norm, tr.rms_norm_fp8):
        with pytest.raises(dla.DLAError) as e:
            call(x.expand(4, 64), w)
        assert e.value.status == dla.DLA_ERR_INVALID_ARG
