"""The gated feed-forward block and its backward pass against their formulas in float64; sizes around
the tiles, layouts, and what is refused.

Tolerances, element by element.  A float32 sum of K products is off by at most K 2^-24 of the sum of
their magnitudes; of float32 inputs, three terms of 8 bits each and the products left out, by 2^-22 of it
more.  silu and its slope are off by (8 + 2 |g|) 2^-24 of |g| and of 1.1, and by what g is off.  Of bfloat16
inputs dg and du are rounded by 2^-8 of themselves (|silu''| <= 0.5); every output is rounded once, g and u as
float32.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U = 2.0 ** -24


def _block():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import block
    return block


def make(N, D, F, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + N + 3 * D + 7 * F)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(DT[dtype])  # noqa: E731
    return rnd(N, D), rnd(F, D) / D ** 0.5, rnd(F, D) / D ** 0.5, rnd(N, F)


def call(block, x, wg, wu, dy, **kw):
    y, parts = block.gated_ff(x, wg, wu, want_parts=True, **kw)
    return (y, parts, *block.gated_ff_backward(x, wg, wu, parts, dy, **kw))


def close(got, want, off, half):
    got = got.double()
    assert torch.isfinite(got).all()
    off = off + 2.0 ** -120
    bad = (got - want).abs() > off + 1.001 * half * (want.abs() + off)
    assert not bad.any(), ((got - want).abs() / (off + half * want.abs())).max()


def check(got, x, wg, wu, dy, dtype):
    y, parts, dx, dwg, dwu = got
    half, f32 = HALF[dtype], dtype == "f32"
    X, G, U_, DY = (t.double() for t in (x, wg, wu, dy))
    N, D, F = X.shape[0], X.shape[1], G.shape[0]
    mm = lambda a, b: a @ b  # noqa: E731
    rel = lambda K: (K + 8) * U + (2.0 ** -22 if f32 else 0)  # noqa: E731
    g, u = mm(X, G.t().contiguous()), mm(X, U_.t().contiguous())
    ag, au = mm(X.abs(), G.abs().t().contiguous()) * rel(D), mm(X.abs(), U_.abs().t().contiguous()) * rel(D)
    q = torch.sigmoid(g)
    silu, slope = g * q, q * (1 + g * (1 - q))
    ulp = (10 + 2 * g.abs()) * U
    close(y, silu * u, 1.1 * ag * u.abs() + silu.abs() * au + ag * au + ulp * (silu * u).abs(), half)
    close(parts[0], g, ag, U)
    close(parts[1], u, au, U)
    dg, du = DY * u * slope, DY * silu
    edg = DY.abs() * (au * (slope.abs() + 0.5 * ag) + u.abs() * (0.5 * ag + 2 * ulp))
    edu = DY.abs() * (1.1 * ag + ulp * silu.abs())
    edg, edu = edg + half * (dg.abs() + edg), edu + half * (du.abs() + edu)
    mdg, mdu = dg.abs() + edg, du.abs() + edu
    close(dx, mm(dg, G) + mm(du, U_),
          mm(edg, G.abs()) + mm(edu, U_.abs()) + rel(2 * F) * (mm(mdg, G.abs()) + mm(mdu, U_.abs())), half)
    t = lambda a: a.t().contiguous()  # noqa: E731
    close(dwg, mm(t(dg), X), mm(t(edg), X.abs()) + rel(N) * mm(t(mdg), X.abs()), half)
    close(dwu, mm(t(du), X), mm(t(edu), X.abs()) + rel(N) * mm(t(mdu), X.abs()), half)


@pytest.mark.parametrize("N,D,F", [(1, 1, 1), (1, 2048, 300), (2, 7, 9), (16, 64, 16), (17, 100, 33), (48, 513, 257), (64, 256, 520),
                                   (65, 8, 8), (65, 64, 64), (100, 96, 200), (128, 128, 128), (129, 72, 136), (130, 65, 67),
                                   (300, 1000, 264), (513, 40, 1030), (1000, 264, 56)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sizes(N, D, F, dtype):
    block = _block()
    ins = make(N, D, F, dtype)
    check(call(block, *ins), *ins, dtype)


@pytest.mark.parametrize("N,D,F,dtype", [(4100, 520, 1544, "bf16"), (3500, 1100, 2500, "bf16"), (2900, 264, 2100, "f32"),
                                         (8200, 2048, 264, "bf16")])
def test_large_tiles(N, D, F, dtype):
    """Sizes past a multiple of the large tiles, for which enough of them are there."""
    block = _block()
    ins = make(N, D, F, dtype)
    check(call(block, *ins), *ins, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [3, 200])
def test_layouts(N, dtype):
    """Padded rows, rows at any element, weights of two strides, a shared projection's halves, broadcast rows."""
    block = _block()
    x, wg, wu, dy = make(N, 72, 40, dtype)
    want = call(block, x, wg, wu, dy)
    pad = lambda t, a, b: torch.nn.functional.pad(t, (a, b), value=float("nan"))[:, a:a + t.shape[1]]  # noqa: E731
    both = torch.cat([wg, wu])
    for v in ((pad(x, 0, 8), wg, wu, pad(dy, 1, 2)), (pad(x, 1, 0), pad(wg, 3, 4), wu, dy), (x, both[:40], both[40:], dy),
              (x, pad(wg, 8, 8), pad(wu, 0, 8), pad(dy, 8, 0))):
        got = call(block, *v)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    out = torch.full((N, 50), 3.0, dtype=DT[dtype], device="cuda")
    block.gated_ff(x, wg, wu, out=out[:, 5:45])
    assert torch.equal(out[:, 5:45], want[0]) and (out[:, :5] == 3).all() and (out[:, 45:] == 3).all()
    one = x[:1].expand(N, -1)
    assert torch.equal(block.gated_ff(one, wg, wu)[0], block.gated_ff(one.contiguous(), wg, wu)[0])


def test_what_lies_around_is_not_read():
    """NaN between the rows' ends and the next rows, and behind the last one, in memory of the call's own."""
    block = _block()
    for N, D, F in ((70, 40, 24), (200, 200, 72)):
        x, wg, wu, dy = make(N, D, F, "bf16")
        want = call(block, x, wg, wu, dy)

        def inside(t):
            a = torch.full((t.shape[0] + 300, t.shape[1] + 24), float("nan"), dtype=t.dtype, device="cuda")
            a[:t.shape[0], :t.shape[1]] = t
            return a[:t.shape[0], :t.shape[1]]

        for a, b in zip(call(block, *(inside(t) for t in (x, wg, wu, dy))), want):
            assert torch.equal(a, b)


def test_gradient_against_differences():
    """Float32 outputs are off by some 1e-6 of their size; over 2 h = 2^-4, of 24 x 30 outputs against
    gradients of order one, by 1e-4, and the third derivative by h^2 / 6 = 2e-4 times a few."""
    block = _block()
    x, wg, wu, dy = make(24, 20, 30, "f32")
    dy = dy / 10
    _, _, *grads = call(block, x, wg, wu, dy)
    gen, h = torch.Generator(device="cuda").manual_seed(1), 2.0 ** -5
    for i, g in enumerate(grads):
        for _ in range(3):
            d = torch.randn(g.shape, generator=gen, device="cuda")
            d /= d.norm()
            at = lambda s: (block.gated_ff(*[t + s * d if j == i else t for j, t in enumerate((x, wg, wu))])[0]  # noqa: E731
                            .double() * dy.double()).sum()
            assert abs((g.double() * d.double()).sum() - (at(h) - at(-h)) / (2 * h)) < 4e-3


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_streams_and_graph(dtype):
    block = _block()
    for N, D, F in ((5, 200, 100), (700, 328, 520), (4100, 520, 1544)):
        x, wg, wu, dy = make(N, D, F, dtype)
        ws = torch.empty(block.gated_ff_workspace_bytes(N, D, F, DT[dtype], backward=True), dtype=torch.uint8, device="cuda")
        a = call(block, x, wg, wu, dy, workspace=ws)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            b = call(block, x, wg, wu, dy)
        stream.synchronize()
        for p, q in zip(a, b):
            assert torch.equal(p, q)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c = call(block, x, wg, wu, dy, workspace=ws)
        for i in range(3):
            x.copy_(torch.randn(x.shape, device="cuda"))
            want = call(block, x, wg, wu, dy)
            graph.replay()
            torch.cuda.synchronize()
            for p, q in zip(want, c):
                assert torch.equal(p, q)


def test_float32_range():
    """Values of very different sizes in one product: float32's precision, not bfloat16's."""
    block = _block()
    x, wg, wu, dy = make(70, 64, 48, "f32")
    s = torch.exp2(torch.randint(-20, 20, (64,), device="cuda").float())
    check(call(block, x * s, wg / s, wu / s, dy), x * s, wg / s, wu / s, dy, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,F", [(16, 24), (1, 1), (300, 521), (4096, 2100)])
def test_empty(D, F, dtype):
    """No rows: weight gradients of zeros, also where their memory held something else."""
    block = _block()
    x, wg, wu, dy = make(0, D, F, dtype)
    torch.full((2, F, D), float("nan"), dtype=DT[dtype], device="cuda")
    y, parts, dx, dwg, dwu = call(block, x, wg, wu, dy)
    assert y.shape == (0, F) and dx.shape == (0, D) and parts.shape == (2, 0, F)
    for t in (dwg, dwu):
        assert torch.equal(t, torch.zeros_like(t))
