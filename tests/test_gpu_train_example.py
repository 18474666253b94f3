"""The training operators together: the differentiable functions against direct calls, and
the example, which has to learn associative recall (a guess among 32 values costs ln 32 =
3.47; an answer known to nine parts in ten less than 0.5) and to answer token by token as
it does over whole sequences, but for its norms' 8 bits (2^-4 of a value at most each)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _train():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import train
    return train


@pytest.mark.parametrize("states", ["f32", "fp8"])
def test_example_learns(states):
    _train()
    from paper_2606_10650_amd import train_example
    losses, off, same = train_example.main(300, states, say=lambda s: None)
    assert losses[0] > 3.0 and sum(losses[-20:]) / 20 < 0.5
    assert off < 0.15 and same > 0.9


def test_recurrence_function():
    tr = _train()
    gen = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    q, k = rnd(2, 2, 90, 64) / 8, rnd(2, 2, 90, 64) / 8
    v, S = rnd(2, 4, 90, 64), rnd(2, 4, 64, 64) / 8
    g = -0.1 * rnd(2, 4, 90).abs()
    ins = [x.requires_grad_() for x in (q, k, v, g, S)]
    do, dS = rnd(2, 4, 90, 64), rnd(2, 4, 64, 64)
    for use_out, use_state in ((1, 1), (1, 0), (0, 1)):
        for x in ins:
            x.grad = None
        out, last = tr.Recurrence.apply(q, k, v, g, S, 0.5, None)
        # a gradient with its last axis strided, and one broadcast
        loss = use_out * (out.transpose(2, 3) * do.transpose(2, 3)).sum() + use_state * (last * dS).sum()
        if not use_out:
            loss = (last * dS).sum()
        if not use_state:
            loss = (out * do).sum()
        loss.backward()
        with torch.no_grad():
            want = tr.recurrence_backward(q, k, v, g, do if use_out else torch.zeros_like(do), scale=0.5, state=S,
                                          dstate=dS if use_state else None)
        for x, y in zip(ins, want):
            assert torch.equal(x.grad, y)
    out, _ = tr.Recurrence.apply(q, k, v, g, S, 0.5, None)
    for x in ins:
        x.grad = None
    out.sum().backward()
    want = tr.recurrence_backward(q.detach(), k.detach(), v.detach(), g.detach(), torch.ones_like(do), scale=0.5,
                                  state=S.detach())
    assert torch.equal(v.grad, want[2])


def test_norm_function():
    tr = _train()
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    x, r, w = (t.requires_grad_() for t in (rnd(2, 7, 100), rnd(2, 7, 100), rnd(100)))
    dy, dh = rnd(2, 7, 100), rnd(2, 7, 100)
    for use_h in (True, False):
        for t in (x, r, w):
            t.grad = None
        y, h = tr.RMSNorm.apply(x, r, w)
        ((y * dy).sum() + ((h * dh).sum() if use_h else 0)).backward()
        got = [x.grad, r.grad, w.grad]
        X, R, W = (t.detach().double().requires_grad_() for t in (x, r, w))
        H = X + R
        Y = H / (H.square().mean(-1, keepdim=True) + 1e-6).sqrt() * W
        ((Y * dy).sum() + ((H * dh).sum() if use_h else 0)).backward()
        for a, b in zip(got, (X.grad, R.grad, W.grad)):
            assert (a.double() - b).norm() <= 1e-5 * b.norm()
