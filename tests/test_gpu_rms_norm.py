"""The residual root-mean-square norm, its 8-bit output and its backward pass against
their formulas in float64; and the calls they refuse.

Tolerances, relative to the reference's norm: float32 sums of D squares, all of one sign,
are off by at most D 2^-24 in any order and by sqrt(D) 2^-24 in a tree's: 1e-5 holds for
D <= 16384 with room.  bfloat16 outputs are rounded once (2^-8: eight significant bits).
The backward pass starts from the stored h: against the formula on that h the same
tolerances hold, dx's relative to the two terms whose difference it is (in a row of one
value they are equal).  An 8-bit value
is off by at most 2^-4 of itself or 2^-10 of the row's scale, times its position's rounding.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
TOL = {"bf16": 2.0 ** -8 + 1e-5, "f32": 1e-5}
SHAPES = [(1, 1), (3, 2), (5, 7), (1, 64), (33, 65), (4, 511), (7, 512), (2, 1000), (1500, 1531), (1100, 2048),
          (9, 2049), (3, 4096), (2, 8195), (5, 16384), (2000, 96)]


def _train():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import train
    return train


def make(N, D, dtype, seed=0, spread=False):
    gen = torch.Generator(device="cuda").manual_seed(seed + N * 7 + D)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    x, r = rnd(N, D), 2 * rnd(N, D)
    if spread:
        x *= torch.exp(3 * rnd(N, 1))
    return x.to(DT[dtype]), r.to(DT[dtype]), (1 + 0.2 * rnd(D)).to(DT[dtype]), rnd(N, D).to(DT[dtype]), \
        rnd(N, D).to(DT[dtype])


def close(got, want, tol, terms=0.0):
    assert torch.isfinite(got.double()).all()
    err, norm = (got.double() - want).norm().item(), want.norm().item() + float(terms)
    assert err <= tol * norm + 1e-30, (err / max(norm, 1e-30), tol)


@pytest.mark.parametrize("N,D", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [True, False])
def test_forward_and_backward(N, D, dtype, residual):
    tr = _train()
    x, r, w, dy, dres = make(N, D, dtype, spread=True)
    eps = 1e-5
    y, h, rstd = tr.rms_norm(x, w, r if residual else None, eps=eps)
    H = x.double() + (r.double() if residual else 0)
    R = 1 / (H.square().mean(-1, keepdim=True) + eps).sqrt()
    close(y, H * R * w.double(), TOL[dtype])
    close(rstd, R[:, 0], 1e-5)
    close(h, H, TOL[dtype])
    if not residual:
        assert h is x
    dx, dw = tr.rms_norm_backward(dy, h, w, rstd, dres=dres if residual else None)
    H = h.double()
    n, dn = H * rstd.double()[:, None], dy.double() * w.double()
    want = (dn - n * (dn * n).mean(-1, keepdim=True)) * rstd.double()[:, None]
    close(dx, want + (dres.double() if residual else 0), TOL[dtype],
          terms=(dn * rstd.double()[:, None]).norm())
    close(dw, (dy.double() * n).sum(0), 1e-5)


@pytest.mark.parametrize("N,D", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_fp8(N, D, dtype):
    tr = _train()
    x, r, w, _, _ = make(N, D, dtype, spread=True)
    y, h, scale = tr.rms_norm_fp8(x, w, r, eps=1e-6)
    H = x.double() + r.double()
    want = H / (H.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()
    close(scale, want.abs().amax(-1) / 448, 1e-5)
    close(h, H, TOL[dtype])
    got = y.double() * scale.double()[:, None]
    assert ((got - want).abs() <= want.abs() * (2.0 ** -4 + 1e-5) + scale.double()[:, None] * 2.0 ** -10).all()
    assert (y.float().abs().amax(-1) == 448).all()


@pytest.mark.parametrize("D", [64, 777])
def test_fp8_odd_rows(D):
    """A row of zeros, one with an infinity, one with a NaN, one of the least numbers."""
    tr = _train()
    x, r, w, _, _ = make(6, D, "f32")
    r.zero_()
    x[1] = 0
    x[2, D // 2] = float("inf")
    x[3, D - 1] = float("nan")
    x[4] *= 1e-30
    y, h, scale = tr.rms_norm_fp8(x, w, r, eps=1e-6)
    torch.cuda.synchronize()
    assert not y[1].float().any() and scale[1] == 0
    assert torch.isnan(y[3].float()).all() and torch.isnan(scale[3])
    assert torch.isnan(y[2].float()).any()
    want = x[4].double() / 1e-3 * w.double()
    got = y[4].double() * scale[4].double()
    assert (got - want).norm() <= 0.04 * want.norm()
    for i in (0, 5):
        assert torch.isfinite(y[i].float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_and_mixed_weight(dtype):
    """Rows of a wider array, at odd elements; a float32 weight; aliased buffers."""
    tr = _train()
    x, r, w, dy, dres = make(50, 300, dtype)
    wide = torch.full((50, 333), float("nan"), dtype=DT[dtype], device="cuda")
    part = wide[:, 5:305]
    part.copy_(x)
    w32 = w.float() * 1.001
    y, h, rstd = tr.rms_norm(part, w32, r)
    H = x.double() + r.double()
    R = 1 / (H.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    close(y, H * R * w32.double(), TOL[dtype])
    dyw = wide[:, 7:307]
    dyw.copy_(dy)
    dx, dw = tr.rms_norm_backward(dyw, h, w32, rstd, dres=dres)
    again, dw2 = tr.rms_norm_backward(dy, h, w32, rstd, dres=dres)
    assert torch.equal(dx, again) and torch.equal(dw, dw2)


def test_against_differences():
    tr = _train()
    x, r, w, dy, dres = make(4, 130, "f32")
    y, h, rstd = tr.rms_norm(x, w, r, eps=1e-6)
    dx, dw = tr.rms_norm_backward(dy, h, w, rstd, dres=dres)
    gen = torch.Generator(device="cuda").manual_seed(3)

    def loss(x, w):
        H = x + r.double()
        return ((H / (H.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w * dy.double()).sum()
                + (H * dres.double()).sum())

    X, W, e = x.double(), w.double(), 1e-5
    d = torch.randn(x.shape, generator=gen, device="cuda", dtype=torch.float64)
    want = (loss(X + e * d, W) - loss(X - e * d, W)) / (2 * e)
    assert abs((dx.double() * d).sum() - want) <= 1e-5 * dx.double().norm() * 4 + 1e-6 * abs(want)
    d = torch.randn(w.shape, generator=gen, device="cuda", dtype=torch.float64)
    want = (loss(X, W + e * d) - loss(X, W - e * d)) / (2 * e)
    assert abs((dw.double() * d).sum() - want) <= 1e-5 * dw.double().norm() * 4 + 1e-6 * abs(want)


def test_no_rows_and_refusals():
    tr = _train()
    from paper_2606_10650_amd import dla
    x, r, w, dy, _ = make(4, 64, "bf16")
    y, h, rstd = tr.rms_norm(x[:0], w, r[:0])
    assert y.shape == (0, 64)
    dx, dw = tr.rms_norm_backward(dy[:0], h, w, rstd)
    torch.cuda.synchronize()
    assert dx.shape == (0, 64) and not dw.any()
    big = torch.zeros((1, 16385), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(dla.DLAError) as e:
        tr.rms_norm(big, big[0])
    assert e.value.status == dla.DLA_ERR_UNSUPPORTED
    with pytest.raises(dla.DLAError) as e:
        tr.rms_norm(x, w, eps=float("nan"))
    assert e.value.status == dla.DLA_ERR_INVALID_ARG
    with pytest.raises(dla.DLAError) as e:
        tr.rms_norm(x[:1].expand(4, 64), w, eps=1e-6) if False else tr.rms_norm(
            x.as_strided((4, 64), (32, 1)), w)      # rows that overlap
    assert e.value.status == dla.DLA_ERR_INVALID_ARG
    with pytest.raises(dla.DLAError) as e:
        tr.rms_norm(x.float(), w)                    # a weight narrower than the rows
    assert e.value.status == dla.DLA_ERR_INVALID_ARG
    for bad in (lambda: tr.rms_norm(x, w[:32]), lambda: tr.rms_norm(x, w, r[:2]),
                lambda: tr.rms_norm(x, w, r.float()), lambda: tr.rms_norm(x.t(), w[:4])):
        with pytest.raises(ValueError):
            bad()
