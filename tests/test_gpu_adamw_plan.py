"""An AdamW plan whose tensors move: gradients made anew, parameters whose data is replaced.
Steps are compared bit by bit with a new plan's over the tensors as they are."""
import pytest
import torch

pytestmark = pytest.mark.gpu

HY = dict(lr=1e-2, betas=(0.9, 0.99), eps=1e-6)


def _train():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import train
    return train


def _rnd(seed, *shape, dtype=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


@pytest.mark.parametrize("states", ["f32", "fp8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_new_gradients_are_taken(states, dtype):
    """Gradients set to None and made anew by the backward pass, some kept alive so that the
    new ones lie elsewhere, beside a gradient that is the caller's own buffer."""
    tr = _train()
    ps = [_rnd(i, 300 + i, dtype=dtype).requires_grad_() for i in range(5)]
    other, buffer = _rnd(9, 100, dtype=dtype), _rnd(10, 100)
    plan = tr.AdamW(states)
    for p in ps:
        p.grad = torch.zeros_like(p)
        plan.add(p, p.grad, weight_decay=0.1)
    plan.add(other, buffer)
    again = [p.detach().clone() for p in ps] + [other.clone()]
    states_ = None
    hold = []
    for t in range(1, 4):
        for i, p in enumerate(ps):
            if t % 2 == 1:
                hold.append(p.grad)
            p.grad = None
        buffer.copy_(_rnd(20 + t, 100))
        sum((p.float() * _rnd(100 * t + i, *p.shape)).sum() for i, p in enumerate(ps)).backward()
        # the step before is done over by a plan of its own, on clones
        fresh = tr.AdamW(states)
        for i, p in enumerate(ps + [other]):
            kw = {} if states_ is None else {k: v for k, v in states_[i].items() if v is not None}
            g = buffer if i == len(ps) else p.grad
            fresh.add(again[i], g.clone(), weight_decay=0.1 if i < len(ps) else 0.0, **kw)
        fresh.step(t, seed=0, **HY)
        plan.step(t, seed=0, **HY)
        states_ = [{k: e[k] for k in ("m", "v", "m_scale", "v_scale")} for e in fresh.kept]
        torch.cuda.synchronize()
        for i, p in enumerate(ps + [other]):
            assert torch.equal(p.detach(), again[i]), (t, i)
            assert torch.equal(plan.kept[i]["m"].view(torch.uint8), fresh.kept[i]["m"].view(torch.uint8))


def test_replaced_data_is_followed():
    """A parameter, a master and a state moved to other memory: the step works there, and
    leaves the old memory alone."""
    tr = _train()
    p, w, g = _rnd(1, 700, dtype=torch.bfloat16), _rnd(2, 700), _rnd(3, 700, dtype=torch.bfloat16)
    plan, other = tr.AdamW(), tr.AdamW()
    p2, w2 = p.clone(), w.clone()
    plan.add(p, g, master=w)
    other.add(p2, g, master=w2)
    plan.step(1, **HY)
    other.step(1, **HY)
    old = [p.data, w.data, plan.kept[0]["v"].data]
    was = [x.clone() for x in old]
    p.data, w.data = p.data.clone(), w.data.clone()
    plan.kept[0]["v"].data = plan.kept[0]["v"].data.clone()
    plan.step(2, **HY)
    other.step(2, **HY)
    torch.cuda.synchronize()
    assert torch.equal(p, p2) and torch.equal(w, w2) and torch.equal(plan.kept[0]["v"], other.kept[0]["v"])
    for x, y in zip(old, was):
        assert torch.equal(x, y)


def test_what_a_step_refuses():
    """A parameter without a gradient, and tensors that no longer fit: an error, and nothing
    changed."""
    tr = _train()
    p = _rnd(1, 64).requires_grad_()
    p.grad = torch.ones_like(p)
    plan = tr.AdamW()
    plan.add(p, p.grad)
    plan.step(1, **HY)
    was = p.detach().clone()
    p.grad = None
    with pytest.raises(ValueError, match="no gradient"):
        plan.step(2, **HY)
    p.grad = torch.ones((128,), device="cuda")[::2]
    with pytest.raises(ValueError):
        plan.step(2, **HY)
    p.grad = torch.ones_like(p)
    q = p.data
    for bad in (q.double(), torch.zeros(65, device="cuda"), q.cpu()):
        p.grad = None
        p.data = bad
        p.grad = torch.ones_like(p)
        with pytest.raises(ValueError):
            plan.step(2, **HY)
    p.grad = None
    p.data = q
    p.grad = torch.ones_like(p)
    torch.cuda.synchronize()
    assert torch.equal(p.detach(), was)
    plan.step(2, **HY)


@pytest.mark.parametrize("factor", [3.402823466e38, -3.401e38])
def test_the_largest_factors_count(factor):
    """A finite grad_scale is one however large: only an infinite one, or NaN, stops the step."""
    tr = _train()
    p, g = torch.ones(64, device="cuda"), torch.full((64,), 2.0 ** -126, device="cuda")
    plan = tr.AdamW()
    plan.add(p, g)
    plan.step(1, lr=0.125, eps=0.0, grad_scale=torch.tensor([factor], device="cuda"))
    torch.cuda.synchronize()
    # the first step is lr in the gradient's direction
    assert ((p - (1 - 0.125 * (1 if factor > 0 else -1))).abs() <= 1e-6).all()


def test_data_replaced_before_the_first_step():
    tr = _train()
    p, g = _rnd(1, 100), _rnd(2, 100)
    plan, other = tr.AdamW(), tr.AdamW()
    plan.add(p, g)
    q = p.clone()
    other.add(q, g)
    p.data = p.data.clone()
    plan.step(1, **HY)
    other.step(1, **HY)
    assert torch.equal(p, q)
    plan = tr.AdamW()
    plan.add(p, g)
    p.data = torch.zeros(50, device="cuda")
    for _ in range(2):
        with pytest.raises(ValueError):
            plan.step(1, **HY)
