"""Decode steps of more heads than a grid dimension takes, against the formula in float32
with float64 sums.  float32: a state is two products and a sum, 2^-22 of their size; an
output's 64 products' sum 1.5e-5 of its norm.  bfloat16 outputs are rounded once, 2^-8."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _train():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import train
    return train


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_step_of_65536_heads(dtype):
    tr = _train()
    B, H, Hk = 2048, 32, 16
    gen = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    q, k = (rnd(B, Hk, 1, 64) / 8).to(dtype), (rnd(B, Hk, 1, 64) / 8).to(dtype)
    v, g, S = rnd(B, H, 1, 64).to(dtype), -rnd(B, H, 1).abs(), rnd(B, H, 64, 64)
    both = lambda x: x.float().repeat_interleave(H // Hk, 1)  # noqa: E731
    want = S * g.exp()[..., None] + both(k).transpose(2, 3) * v.float()
    size = S.abs() * g.exp()[..., None] + (both(k).transpose(2, 3) * v.float()).abs()
    o = (want.double() * both(q).transpose(2, 3)).sum(2, keepdim=True) * 0.5
    out, last = tr.recurrence(q, k, v, g, scale=0.5, state=S, state_out=S)
    torch.cuda.synchronize()
    assert last is S and ((S - want).abs() <= 2.0 ** -22 * size + 1e-30).all()
    tol = 1.5e-5 if dtype == torch.float32 else 2.0 ** -8
    err = (out.double() - o).flatten(2).norm(dim=-1)
    assert (err <= tol * o.flatten(2).norm(dim=-1) + 1e-5).all()


def test_no_tokens_of_65536_heads():
    tr = _train()
    B, H = 2048, 32
    z = torch.zeros((B, H, 0, 64), device="cuda")
    S = torch.randn((B, H, 64, 64), device="cuda")
    _, last = tr.recurrence(z, z, z, torch.zeros((B, H, 0), device="cuda"), state=S, want_state=True)
    assert torch.equal(last, S)
    _, last = tr.recurrence(z, z, z, torch.zeros((B, H, 0), device="cuda"), want_state=True)
    assert not last.any()
