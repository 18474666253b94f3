"""Log probabilities of tokens, entropies, the largest alternatives and the logits' gradient against
their formulas in float64; masks, ties, odd rows; and what is refused.

Tolerances.  With m a row's largest logit and s the sum of the others' exp(l - m): each difference is
off by 2^-24 of itself, its exponential by (2 + 2 |d|) 2^-24, a float32 sum of n terms by n 2^-24 at most
(threads sum V / 64 at most, then 10 pairs), so s by (2 + 2 D + V / 64 + 12) 2^-24 with D = 104, beyond
which terms are below 2^-149.  Of terms p |d| <= 1 / e of the largest matter, so half of that holds for
the entropy with a term more.  tol(V) = (230 + V / 64) 2^-24, absolute, bounds log(1 + s) and entropy
relative to 1 + entropy; the logits' differences add 2^-24 of their size.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U = 2.0 ** -24
INF = math.inf


def tol(V):
    return (230 + V / 64) * U


def _block():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import block
    return block


def make(N, V, dtype, *, masked=0.0, spread=3.0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + 13 * N + V)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    l = spread * rnd(N, V)
    if masked:
        l[torch.rand((N, V), generator=gen, device="cuda") < masked] = -INF
    tok = torch.randint(0, V, (N,), generator=gen, device="cuda")
    tok[torch.rand((N,), generator=gen, device="cuda") < 0.2] = -100
    return l.to(DT[dtype]), tok, rnd(N), rnd(N), rnd(N)


def formula(l, tok):
    """logprob, lse, entropy, log p in float64; rows of -inf alone have no distribution."""
    l = l.double()
    m, at = l.max(-1, keepdim=True)
    d = torch.where(m == -INF, -INF, l - m)
    # (the largest one's term apart: 64 bits too would lose log1p(4 e^-30), and log 5 next to 3e38)
    rest = torch.log1p(d.exp().scatter(1, at, 0.0).sum(-1, keepdim=True))
    lse, logp = m + rest, d - rest
    p = logp.exp()
    ent = torch.where(m == -INF, 0.0, rest)[:, 0] - torch.where(p > 0, p * d, 0.0).sum(-1)
    lp = torch.where(tok >= 0, logp.gather(1, tok.clamp(min=0)[:, None])[:, 0], 0.0)
    return lp, lse[:, 0], ent, logp


def check_forward(block, l, tok, top):
    N, V = l.shape
    lp, lse, ent, ids, tops = block.token_logprobs(l, tok, top=top, entropy=True)
    LP, LSE, ENT, logp = formula(l, tok)
    size = l.double().abs().masked_fill(l == -INF, 0).amax(-1)

    def near(got, want, off):
        got = got.double()
        inf = torch.isinf(want)
        assert torch.equal(got[inf], want[inf])
        assert ((got - want).abs()[~inf] <= off.expand_as(want)[~inf]).all(), ((got - want).abs() / off)[~inf].max()

    # a log probability near zero keeps its digits
    near(lp, LP, tol(V) * LP.abs().clamp(max=1) + 4 * U * (size + LP.abs()) * (LP.abs() > 0.1) + 2.0 ** -126)
    near(lse, LSE, tol(V) + 4 * U * (size + LSE.abs()))
    near(ent, ENT, (2 * tol(V)) * (1 + ENT) + 4 * U * ENT)
    if top:
        order = torch.sort(l.float() + 0.0, dim=-1, descending=True, stable=True)
        assert torch.equal(ids, order.indices[:, :top])
        near(tops, logp.gather(1, ids), tol(V) + 4 * U * (size[:, None] + logp.gather(1, ids).abs()))
    return lp, lse, ent


def check_backward(block, l, tok, lp, lse, ent, dlp, dent, dlse, dtype):
    V = l.shape[1]
    LP, LSE, ENT, logp = formula(l, tok)
    p = logp.exp()
    asked = (tok >= 0)[:, None]
    one = torch.zeros_like(p).scatter_(1, tok.clamp(min=0)[:, None], 1.0) * asked
    row = lambda t: t.double()[:, None]  # noqa: E731
    size = l.double().abs().masked_fill(l == -INF, 0).amax(-1, keepdim=True)
    for a, h, z in ((dlp, None, None), (dlp, dent, None), (None, dent, None), (dlp, dent, dlse), (None, None, dlse)):
        got = block.token_logprobs_backward(l, tok, lp, lse, a, entropy=ent, dentropy=h, dlse=z).double()
        want, mag = torch.zeros_like(p), torch.zeros_like(p)
        if a is not None:
            want = want + row(a) * asked * (one - p)
            mag = mag + (row(a) * asked).abs() * ((1 - p) * one + p)
        if h is not None:
            inner = torch.where(p > 0, logp + ENT[:, None], 0.0)
            want = want - row(h) * p * inner
            mag = mag + row(h).abs() * p * (torch.where(p > 0, logp.abs(), 0.0) + ENT[:, None] + 1)
        if z is not None:
            want = want + row(z) * p
            mag = mag + row(z).abs() * p
        want = torch.where(LSE[:, None] == -INF, 0.0, want)
        off = mag * (2 * tol(V) + 8 * U * (size + 16)) + 2.0 ** -120
        assert ((got - want).abs() <= off + HALF[dtype] * 1.001 * (want.abs() + off)).all()


@pytest.mark.parametrize("N,V", [(1, 1), (3, 2), (4, 7), (33, 64), (5, 1000), (2, 1025), (9, 8191), (3, 32003), (2, 50304),
                                 (2, 65536), (2, 70001), (1, 262145)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("masked", [0.0, 0.9])
def test_forward_and_backward(N, V, dtype, masked):
    block = _block()
    l, tok, dlp, dent, dlse = make(N, V, dtype, masked=masked)
    if masked:
        l[:, V // 2] = 1.0
    for top in {0, 1, min(V, 20), min(V, 64)}:
        out = check_forward(block, l, tok, top)
    check_backward(block, l, tok, *out, dlp, dent, dlse, dtype)


@pytest.mark.parametrize("V", [5, 300, 9000, 70000])
def test_odd_rows(V):
    """All equal, ties between +0 and -0, one logit left, none left, NaN and +inf, a peak, huge values."""
    block = _block()
    l, tok, *_ = make(10, V, "f32")
    tok = torch.randint(0, V, (10,), device="cuda")
    tok[9] = 0
    l[0] = 2.5
    l[1] = 0.0
    l[1, 1::2] = -0.0
    l[2] = -INF
    l[2, tok[2]] = 3.0
    l[3] = -INF
    l[4, 1] = float("nan")
    l[5, V - 1] = INF
    l[6] = -30.0
    l[6, tok[6]] = 0.0           # log p about -V e^-30
    l[7] = 3e38
    l[8] = -3e38
    top = min(V, 64)
    rows = [0, 1, 2, 3, 6, 7, 8, 9]
    lp, lse, ent = check_forward(block, l[rows].contiguous(), tok[rows].contiguous(), top)
    d = torch.ones(8, device="cuda")
    check_backward(block, l[rows].contiguous(), tok[rows].contiguous(), lp, lse, ent, d, d, d, "f32")
    assert lp[2] == 0 and ent[2] == 0 and lp[3] == -INF and ent[3] == 0 and lse[3] == -INF
    lp, lse, ent, ids, tops = block.token_logprobs(l, tok, top=top, entropy=True)
    for r in (4, 5):
        assert torch.isnan(lp[r]) and torch.isnan(ent[r]) and ((ids[r] >= 0) & (ids[r] < V)).all()
        assert torch.isnan(tops[r]).any()
    assert torch.isfinite(lp[9]) and torch.isfinite(ent[9])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [5, 600])
def test_far_from_the_first_logits(dtype, N):
    """Rows whose first logits say nothing of the others: shut out, far below, far above."""
    block = _block()
    l, tok, dlp, dent, dlse = make(N, 20000, dtype)
    l[0, :9000] = -INF
    l[0, 9000:] -= 300
    l[1, :9000] -= 100
    l[2, 9000:] -= 100
    l[3, :] = -INF
    l[3, 19999] = -50.0
    l[4, 9000:] = -INF
    out = check_forward(block, l, tok, 20)
    check_backward(block, l, tok, *out, dlp, dent, dlse, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [2000, 50000, 100000])
def test_many_reach_the_bound(dtype, V):
    """Rising logits, whose largest all lie with few threads, and one value over and over."""
    block = _block()
    l = torch.arange(V, device="cuda", dtype=torch.float32)[None].repeat(3, 1) / V
    l[1] = l[1].flip(0)
    l[2] = (torch.arange(V, device="cuda") % 3 == 0).float()
    check_forward(block, l.to(DT[dtype]), torch.zeros(3, dtype=torch.int64, device="cuda"), 64)


def test_tokens_outside():
    """A negative token asks for nothing; one past the vocabulary gives NaN in its row alone."""
    block = _block()
    l, _, dlp, *_ = make(4, 100, "f32")
    tok = torch.tensor([3, -1, 100, 1 << 40], device="cuda")
    lp, lse, _, _, _ = block.token_logprobs(l, tok)
    assert torch.isfinite(lp[0]) and lp[1] == 0 and torch.isnan(lp[2:]).all() and torch.isfinite(lse).all()
    d = block.token_logprobs_backward(l, tok, lp, lse, dlp)
    assert torch.isfinite(d[0]).all() and not d[1].any() and torch.isnan(d[2:]).all()
    none = block.token_logprobs(l, top=3)
    assert none[0] is None and torch.equal(none[1], lse)


def test_rows_as_they_lie():
    """Padded rows at any element, broadcast rows, the gradient over the logits, and beside it nothing."""
    block = _block()
    l, tok, dlp, dent, _ = make(6, 777, "bf16")
    lp, lse, ent, ids, tops = block.token_logprobs(l, tok, top=5, entropy=True)
    want = block.token_logprobs_backward(l, tok, lp, lse, dlp, entropy=ent, dentropy=dent)
    for off, wide in ((0, 777), (1, 800), (3, 781)):
        w = torch.full((6, wide), 9.0, dtype=torch.bfloat16, device="cuda")
        v = w[:, off:off + 777]
        v.copy_(l)
        got = block.token_logprobs(v, tok, top=5, entropy=True)
        for a, b in zip(got, (lp, lse, ent, ids, tops)):
            assert torch.equal(a, b)
        assert torch.equal(block.token_logprobs_backward(v, tok, lp, lse, dlp, entropy=ent, dentropy=dent, dlogits=v), want)
        assert (w[:, :off] == 9).all() and (w[:, off + 777:] == 9).all()
    one = l[:1].expand(6, -1)
    a, b = block.token_logprobs(one, tok, entropy=True), block.token_logprobs(one.contiguous(), tok, entropy=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])


def test_same_bits_streams_and_graph():
    block = _block()
    for N, V in ((3, 200000), (50, 5000)):
        l, tok, dlp, dent, dlse = make(N, V, "bf16")

        def both():
            o = block.token_logprobs(l, tok, top=20, entropy=True)
            return (*o, block.token_logprobs_backward(l, tok, o[0], o[1], dlp, entropy=o[2], dentropy=dent, dlse=dlse))

        a = both()
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            b = both()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c = both()
        for p, q in zip(a, b):
            assert torch.equal(p, q)
        for i in range(3):
            l.copy_(torch.randn((N, V), device="cuda") * 3)
            want = both()
            graph.replay()
            torch.cuda.synchronize()
            for p, q in zip(want, c):
                assert torch.equal(p, q)


def test_gradient_against_differences():
    """Central differences of float32 losses: outputs are off by some 1e-5 (tol(300) and 2^-22 of their
    size), so differences over 2 h = 2^-4 by 1e-3 and more for the third derivative's h^2 / 6."""
    block = _block()
    l, tok, dlp, dent, dlse = make(4, 300, "f32", spread=1.0)
    out = block.token_logprobs(l, tok, entropy=True)
    g = block.token_logprobs_backward(l, tok, out[0], out[1], dlp, entropy=out[2], dentropy=dent, dlse=dlse)

    def loss(x):
        lp, lse, ent, _, _ = block.token_logprobs(x, tok, entropy=True)
        return (lp * dlp + ent * dent + lse * dlse).double().sum()

    gen, h = torch.Generator(device="cuda").manual_seed(3), 2.0 ** -5
    for _ in range(4):
        d = torch.randn(l.shape, generator=gen, device="cuda")
        d /= d.norm()
        assert abs((g * d).double().sum() - (loss(l + h * d) - loss(l - h * d)) / (2 * h)) < 3e-3


def test_empty():
    block = _block()
    l = torch.zeros((0, 10), device="cuda")
    tok = torch.zeros((0,), dtype=torch.int64, device="cuda")
    lp, lse, ent, ids, tops = block.token_logprobs(l, tok, top=2, entropy=True)
    assert lp.numel() == 0 and ids.shape == (0, 2)
    assert block.token_logprobs_backward(l, tok, lp, lse, lp).shape == (0, 10)
