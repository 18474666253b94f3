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
