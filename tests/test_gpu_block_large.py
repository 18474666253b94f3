"""The operators around the recurrence where elements lie past 2^31, and where rows are more than a launch's workgroups: the
last rows as a call of their own gives them."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _block():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.get_device_properties(0).total_memory < 100e9:
        pytest.skip("100 GB are wanted")
    torch.cuda.empty_cache()
    from paper_2606_10650_amd import block
    return block


def _rnd(*shape, seed=0):
    t = torch.empty(shape, dtype=BF, device="cuda")
    t.normal_(generator=torch.Generator(device="cuda").manual_seed(seed + t.numel() % 1000003))
    return t


def test_short_conv():
    block = _block()
    B, T, C, W = 2, 70000, 16400, 4
    x, dy, w = _rnd(B, T, C), _rnd(B, T, C, seed=1), _rnd(C, W)
    assert x.numel() > 1 << 31
    out, last = block.short_conv(x, w, want_state=True)
    cut = T - 300
    before = x[:, cut - 3:cut].contiguous()
    want, state = block.short_conv(x[:, cut:], w, state=before, want_state=True)
    assert torch.equal(out[:, cut:], want) and torch.equal(last, state)
    del out
    dy[:, :cut] = 0        # so the weights' gradient is the last tokens'
    dx, dw, _, _ = block.short_conv_backward(x, w, dy)
    tail, dwt, _, ds = block.short_conv_backward(x[:, cut:], w, dy[:, cut:].contiguous(), state=before)
    assert torch.equal(dx[:, cut:], tail) and torch.equal(dx[:, cut - 3:cut], ds) and not dx[:, :cut - 3].any()
    # float32 sums of 600 products in another order: 600 2^-24 of their magnitudes, which are some sqrt(600) times the sum
    assert (dw - dwt).norm() <= 600 ** 1.5 * 2.0 ** -24 * dwt.norm()


def test_gated_norm():
    block = _block()
    N, D = (1 << 20) + 77, 2048
    x, gate, res, dh, dy = (_rnd(N, D, seed=i) for i in range(5))
    w, w2 = _rnd(D), _rnd(D, seed=9)
    assert x.numel() > 1 << 31
    whole = block.gated_norm(x, w, gate, res, scale=0.5, next_weight=w2)
    cut = slice(N - 50, N)
    own = block.gated_norm(x[cut], w, gate[cut], res[cut], scale=0.5, next_weight=w2)
    for a, b in zip(whole, own):
        assert torch.equal(a[cut], b)
    back = lambda s, h: block.gated_norm_backward(dh[s], x[s], w, h[2], gate[s], res[s], scale=0.5, next_weight=w2, dy=dy[s], y_rstd=h[3])  # noqa: E731
    for a, b in zip(back(slice(0, N), whole)[:3], back(cut, own)[:3]):
        assert torch.equal(a[cut], b)


def test_log_probabilities():
    block = _block()
    N, V = 45000, 50304
    l = _rnd(N, V)
    assert l.numel() > 1 << 31
    tok = torch.randint(0, V, (N,), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    cut = slice(N - 600, N)        # (600 rows are not worked on in parts either)
    whole, own = (block.token_logprobs(l[s], tok[s], top=3, entropy=True) for s in (slice(0, N), cut))
    for a, b in zip(whole, own):
        assert torch.equal(a[cut], b)
    f = torch.ones(N, device="cuda")
    back = lambda s, v: block.token_logprobs_backward(l[s], tok[s], v[0], v[1], f[s], entropy=v[2], dentropy=f[s])  # noqa: E731
    assert torch.equal(back(slice(0, N), whole)[cut], back(cut, own))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_rows_than_workgroups(dtype):
    """2^20 workgroups forward; each row by itself against the formula in float64, off by some 2^-22 of order one."""
    block = _block()
    N, V = (1 << 20) + 1234, 9
    l = _rnd(N, V) if dtype == "bf16" else _rnd(N, V).float()
    tok = torch.randint(0, V, (N,), device="cuda")
    lp, lse, ent, ids, tops = block.token_logprobs(l, tok, top=2, entropy=True)
    logp = torch.log_softmax(l.double(), -1)
    assert (lp - logp.gather(1, tok[:, None])[:, 0]).abs().max() < 2e-6
    assert (lse - torch.logsumexp(l.double(), -1)).abs().max() < 2e-6 and (ent + (logp.exp() * logp).sum(-1)).abs().max() < 4e-6
    assert (tops - logp.gather(1, ids)).abs().max() < 2e-6 and (tops[:, 0] - logp.amax(-1)).abs().max() < 2e-6


def test_feed_forward():
    block = _block()
    N, D, F = 300000, 64, 7300
    x, wg, wu = _rnd(N, D), _rnd(F, D) / 8, _rnd(F, D, seed=1) / 8
    cut = slice(N - 1000, N)
    y, parts = block.gated_ff(x, wg, wu, want_parts=True)
    assert y.numel() > 1 << 31
    own, own_parts = block.gated_ff(x[cut], wg, wu, want_parts=True)
    assert torch.equal(y[cut], own) and torch.equal(parts[:, cut], own_parts)
    del y
    dy = torch.zeros((N, F), dtype=BF, device="cuda")
    dy[cut] = _rnd(1000, F)
    dx, dwg, dwu = block.gated_ff_backward(x, wg, wu, parts, dy)
    wx, wwg, wwu = block.gated_ff_backward(x[cut], wg, wu, own_parts, dy[cut].contiguous())
    assert not dx[:N - 1000].any()
    # the same products in sums of another order, each rounded once to bfloat16
    for a, b in ((dx[cut], wx), (dwg, wwg), (dwu, wwu)):
        assert (a.double() - b.double()).norm() <= 2.0 ** -8 * b.double().norm()
