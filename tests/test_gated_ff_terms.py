"""Float32 in the feed-forward block: every term of both operands is in the products, and what infinities give.

A float32 value is the sum of three bfloat16 terms, and a product of two the sum of six of terms' products.  In a sum of
hundreds of products a lost term, at most 2^-17 of one of them, is no more than what rounding may do; so each sum here
has one product that is not zero, or a few: of x's rows, or of the weights', one value each, at every place of K.

Bounds, element by element.  A sum of c products that are not zero is off by (c + 8) U + 2^-22 of their magnitudes
(U = 2^-24; adding zeros is exact), silu and its slope by what a sigmoid's (5 + 1.3 |g| (1 - s)) U makes of them.  Without
a GPU: the same products formed from the terms are inside these bounds, and outside without any one pair of terms."""
import pytest
import torch

U = 2.0 ** -24
PAIRS = [(2, 0), (0, 2), (1, 1), (1, 0), (0, 1), (0, 0)]


def make(N, D, F, sparse, device="cpu"):
    gen = torch.Generator().manual_seed(N + 3 * D + 7 * F)
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    def one(t):
        """One value of each row, those of neighbouring rows far apart."""
        n, K = t.shape
        at = (torch.arange(n) * next(p for p in (7919, 7907, 7901) if K % p) + n // 3) % K
        return torch.zeros_like(t).scatter_(1, at[:, None], t.gather(1, at[:, None]))
    x, wg, wu = rnd(N, D), 0.3 * rnd(F, D), rnd(F, D)
    if sparse == "x":
        x = one(x)
    else:
        wg, wu = one(wg), one(wu)
    return [t.to(device) for t in (x, wg, wu, rnd(N, F))]


def _mm(a, b):
    return a @ b.contiguous()


def wanted(x, wg, wu, dy):
    """{name: (value in float64, bound)}"""
    X, G, W, DY = (t.double() for t in (x, wg, wu, dy))
    nz = lambda t: (t != 0).double()  # noqa: E731
    rel = lambda a, b: (_mm(nz(a), nz(b)) + 8) * U + 2.0 ** -22  # noqa: E731
    size = lambda a, b: _mm(a.abs(), b.abs())  # noqa: E731
    g, u = _mm(X, G.t()), _mm(X, W.t())
    ag, au = size(X, G.t()) * rel(X, G.t()), size(X, W.t()) * rel(X, W.t())
    q = torch.sigmoid(g)
    silu, slope = g * q, q * (1 + g * (1 - q))
    es = (5 + 1.3 * g.abs() * (1 - q)) * U
    eslope = q * (es * (1 + g * (1 - q)).abs() + g.abs() * (q * es + U) + 3 * U * (1 + g.abs() * (1 - q))) + 0.5 * ag
    esilu = silu.abs() * (es + 2 * U) + 1.1 * ag
    y = silu * u
    ey = esilu * u.abs() + silu.abs() * au + esilu * au + 2 * U * y.abs()
    dg, du = DY * u * slope, DY * silu
    edg = DY.abs() * (au * (slope.abs() + eslope) + u.abs() * eslope) + 3 * U * dg.abs()
    edu = DY.abs() * esilu + 2 * U * du.abs()
    mg, mu = dg.abs() + edg, du.abs() + edu
    dx = _mm(dg, G) + _mm(du, W)
    edx = size(edg, G) + size(edu, W) + (rel(dg, G) + rel(du, W)) * (size(mg, G) + size(mu, W))
    t = lambda a: a.t()  # noqa: E731
    dwg, dwu = _mm(t(dg), X), _mm(t(du), X)
    r = rel(t(dg), X)
    return {"g": (g, ag), "u": (u, au), "y": (y, ey), "dx": (dx, edx), "dwg": (dwg, size(t(edg), X) + r * size(t(mg), X)),
            "dwu": (dwu, size(t(edu), X) + r * size(t(mu), X))}


def wrong(got, want):
    bad = []
    for k, (v, e) in want.items():
        t = got[k].double()
        if not torch.isfinite(t).all() or not ((t - v).abs() <= e + 1.001 * U * (v.abs() + e) + 2.0 ** -120).all():
            bad.append(k)
    return bad


def by_terms(x, wg, wu, dy, lost=None):
    """The block's results with its products formed from the terms; lost: (a kind of product, a pair left out)."""
    def terms(v):
        a = v.bfloat16()
        b = (v - a.float()).bfloat16()
        return [t.double() for t in (a, b, (v - a.float() - b.float()).bfloat16())]
    def product(kind, a, b):
        a, b = terms(a), terms(b)
        return sum(_mm(a[i], b[j]) for i, j in PAIRS if lost != (kind, (i, j)))
    g, u = (product(0, x, w.t()).float() for w in (wg, wu))
    q = torch.sigmoid(g.double())
    dg, du = (dy * u * q * (1 + g * (1 - q))).float(), (dy * g * q).float()
    return dict(g=g, u=u, y=(g * q * u).float(), dx=(product(1, dg, wg) + product(1, du, wu)).float(),
                dwg=product(2, dg.t(), x).float(), dwu=product(2, du.t(), x).float())


@pytest.mark.parametrize("N,D,F", [(70, 300, 130), (300, 300, 300), (150, 64, 257)])
def test_bounds_tell(N, D, F):
    for sparse, kinds in (("x", {0: ("g", "u"), 2: ("dwg", "dwu")}), ("w", {0: ("g", "u"), 1: ("dx",)})):
        ins = make(N, D, F, sparse)
        want = wanted(*ins)
        assert wrong(by_terms(*ins), want) == []
        for kind, names in kinds.items():
            for pair in PAIRS:
                assert set(names) <= set(wrong(by_terms(*ins, lost=(kind, pair)), want)), (sparse, kind, pair)


@pytest.mark.gpu
@pytest.mark.parametrize("sparse", ["x", "w"])
@pytest.mark.parametrize("N,D,F", [(1, 300, 40), (16, 130, 64), (64, 300, 257), (65, 300, 130), (300, 300, 300), (150, 64, 257), (1531, 321, 1000),
                                   (700, 1000, 264), (2900, 264, 2100), (4130, 1280, 154)])
def test_every_term(N, D, F, sparse):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import block
    x, wg, wu, dy = ins = make(N, D, F, sparse, "cuda")
    y, parts = block.gated_ff(x, wg, wu, want_parts=True)
    dx, dwg, dwu = block.gated_ff_backward(x, wg, wu, parts, dy)
    assert wrong(dict(g=parts[0], u=parts[1], y=y, dx=dx, dwg=dwg, dwu=dwu), wanted(*ins)) == []


@pytest.mark.gpu
@pytest.mark.parametrize("N", [3, 64, 65, 200])
def test_infinities(N):
    """Up to 64 rows an infinity gives what float32's own sums give.  Of more rows it is an infinity or NaN, in the same places;
    and the rows and columns without one are as they were."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import block
    gen = torch.Generator(device="cuda").manual_seed(N)
    x, wg, wu = (torch.randn(s, generator=gen, device="cuda") for s in ((N, 40), (72, 40), (72, 40)))
    want = block.gated_ff(x, wg, wu)[0]
    x[1, 7], wu[5, 3] = float("inf"), float("-inf")
    y, parts = block.gated_ff(x, wg, wu, want_parts=True)
    touched = torch.zeros_like(y, dtype=torch.bool)
    touched[1], touched[:, 5] = True, True
    assert torch.equal(y[~touched], want[~touched])
    g, u = x.cpu().double() @ wg.cpu().double().t(), x.cpu().double() @ wu.cpu().double().t()
    for got, w in zip(parts.cpu(), (g, u)):
        assert torch.equal(torch.isfinite(got), torch.isfinite(w))
        if N <= 64:
            assert torch.equal(got.isnan(), w.isnan()) and torch.equal(got[got.isinf()].double(), w[w.isinf()])
