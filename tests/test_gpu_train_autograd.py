"""The differentiable functions with the gradients that torch hands them in earnest, and
what they refuse."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _train():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import train
    return train


def _recurrence_inputs(T=40, dtype=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(T)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    q, k, v, S = rnd(1, 2, T, 64) / 8, rnd(1, 2, T, 64) / 8, rnd(1, 2, T, 64), rnd(1, 2, 64, 64) / 8
    g = -0.1 * rnd(1, 2, T).abs()
    return [x.requires_grad_() for x in (q.to(dtype), k.to(dtype), v.to(dtype), g, S)]


def _norm_inputs(N=6, D=96):
    gen = torch.Generator(device="cuda").manual_seed(N * D)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    return [x.requires_grad_() for x in (rnd(N, D), rnd(N, D), 1 + 0.1 * rnd(D))]


def test_second_derivatives_are_refused():
    tr = _train()
    x, r, w = _norm_inputs()
    y, h = tr.RMSNorm.apply(x.tanh(), r, w)
    (g,) = torch.autograd.grad((y ** 3).sum() + h.sin().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.square().sum().backward()
    ins = _recurrence_inputs()
    out, last = tr.Recurrence.apply(*ins, 1.0, None)
    (g,) = torch.autograd.grad((out ** 3).sum() + (last ** 3).sum(), ins[0], create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.square().sum().backward()


def _norm64(x, r, w):
    h = x + r
    return h / (h.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w, h


@pytest.mark.parametrize("loss", [
    lambda y, h: y.sum(),                                       # one number for all
    lambda y, h: y.mean() + h.mean(),
    lambda y, h: (y.sum(0) * torch.arange(96, device="cuda")).sum() + h.sum(1)[0],   # one row for all tokens
    lambda y, h: (y.sum(1) * torch.arange(6, device="cuda")).sum(),                  # one number a row
    lambda y, h: (y.t() * torch.arange(6, device="cuda")).sin().sum(),               # transposed
    lambda y, h: torch.cat([torch.zeros(3, device="cuda"), y.flatten(), h.flatten()]).cos().sum(),
], ids=["sum", "mean", "tokens", "rows", "transposed", "cat"])
def test_norm_takes_any_gradient(loss):
    tr = _train()
    ins = _norm_inputs()
    loss(*tr.RMSNorm.apply(*ins)).backward()
    exact = [x.detach().double().requires_grad_() for x in ins]
    loss(*_norm64(*exact)).backward()
    for x, e in zip(ins, exact):
        # cos and sin turn 1e-5 of their argument into as much of themselves at most
        assert (x.grad.double() - e.grad).norm() <= 4e-5 * e.grad.norm() + 1e-6


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shift", [1, 2, 5])
def test_recurrence_takes_gradients_at_any_address(shift, dtype):
    """The gradients of `out` and of the last state as views of a longer vector's, at odd
    elements: the same bits as from tensors of their own."""
    tr = _train()
    ins = _recurrence_inputs(dtype=dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda x: torch.randn(x.shape, generator=gen, device="cuda").to(x.dtype)  # noqa: E731
    pad = torch.zeros(shift, device="cuda")
    out, last = tr.Recurrence.apply(*ins, 0.5, None)
    do, dS = rnd(out), rnd(last)
    # each cat's backward pass hands out a narrow part of its gradient
    loss = (torch.cat([pad.to(dtype), out.flatten()]) * torch.cat([pad.to(dtype), do.flatten()])).sum() + \
        (torch.cat([pad, last.flatten()]) * torch.cat([pad, dS.flatten()])).sum()
    loss.backward()
    with torch.no_grad():
        want = tr.recurrence_backward(*ins[:4], do, scale=0.5, state=ins[4], dstate=dS)
    for x, y in zip(ins, want):
        assert torch.equal(x.grad, y.to(x.dtype))


def test_recurrence_takes_broadcast_gradients():
    tr = _train()
    ins = _recurrence_inputs()
    out, last = tr.Recurrence.apply(*ins, 0.5, None)
    (out.sum(2).sum() + 2 * last.sum()).backward()
    with torch.no_grad():
        want = tr.recurrence_backward(*ins[:4], torch.ones_like(out), scale=0.5, state=ins[4],
                                      dstate=torch.full_like(last, 2.0))
    for x, y in zip(ins, want):
        assert torch.equal(x.grad, y)


def test_norm_takes_broadcast_inputs():
    """One row for all tokens, as x, as the residual, and transposed ones: the gradient is
    summed over what it was broadcast to."""
    tr = _train()
    x, r, w = _norm_inputs()
    dy = torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    row = x.detach()[0].clone().requires_grad_()
    turned = x.detach().t().contiguous().requires_grad_()
    for a, b, leaf in ((row.expand(6, 96), r, row), (r, row.expand(6, 96), row), (turned.t(), r, turned)):
        leaf.grad = None
        (tr.RMSNorm.apply(a, b, w)[0] * dy).sum().backward()
        L = leaf.detach().double().requires_grad_()
        wide = L.t() if leaf is turned else L.expand(6, 96)
        (_norm64(*((wide, r.detach().double()) if a is not r else (r.detach().double(), wide)),
                 w.detach().double())[0] * dy).sum().backward()
        assert (leaf.grad.double() - L.grad).norm() <= 1e-5 * L.grad.norm()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("use_h", [False, True])
def test_norm_without_a_residual(use_h, dtype):
    """h is x itself; the gradients are those of x as the residual of zeros, bit by bit."""
    tr = _train()
    x, _, w = (t.detach().to(dtype).requires_grad_() for t in _norm_inputs())
    gen = torch.Generator(device="cuda").manual_seed(8)
    dy, dh = (torch.randn(x.shape, generator=gen, device="cuda").to(dtype) for _ in range(2))
    got = []
    for a, b in ((x, None), (torch.zeros_like(x), x)):
        x.grad = w.grad = None
        y, h = tr.RMSNorm.apply(a, b, w)
        assert torch.equal(h, x)
        ((y * dy).sum() + ((h * dh).sum() if use_h else 0)).backward()
        got.append((y.detach(), x.grad, w.grad))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    # h stands for x in what follows it
    with torch.no_grad():
        y, h = tr.RMSNorm.apply(x.detach().view(2, 3, 96), None, w.detach())
        assert y.shape == h.shape == (2, 3, 96) and h.data_ptr() == x.data_ptr()


def test_tensors_in_host_memory_are_refused():
    tr = _train()
    q, g, x, w = torch.zeros(1, 1, 4, 64), torch.zeros(1, 1, 4), torch.zeros(4, 64), torch.ones(64)
    plan = tr.AdamW()
    plan.add(w, torch.ones(64))
    for bad in (lambda: tr.recurrence(q, q, q, g), lambda: tr.recurrence_backward(q, q, q, g, q),
                lambda: tr.rms_norm(x, w), lambda: tr.rms_norm_fp8(x, w),
                lambda: tr.rms_norm_backward(x, x, w, torch.ones(4)), lambda: plan.step(1, lr=1e-3)):
        with pytest.raises(ValueError, match="cuda device"):
            bad()
