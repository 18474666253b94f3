"""AdamW's 8-bit states bit by bit: codes and scales against the float32 operations that
dla_train.h lists, done by numpy on the host."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F = np.float32
BETAS = (0.9, 0.995)


def _train():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import train
    return train


def _uniform(n, number, seed):
    low = np.uint64(0xFFFFFFFF)
    h = (np.arange(n, dtype=np.uint64) + np.uint64(0x9E3779B9 * (number + 1)) & low) ^ np.uint64(seed)
    h = h * np.uint64(0x2545F491) & low
    h ^= h >> np.uint64(16)
    h = h * np.uint64(0x9E3779B1) & low
    h ^= h >> np.uint64(15)
    return (h >> np.uint64(16)).astype(F) / F(65536), (h & np.uint64(65535)).astype(F) / F(65536)


def _values(code, scale):
    return code.float().numpy() * np.repeat(scale, 256)[:len(code)]


def _code(x, u, root):
    """Codes and scales of x; u: None for the nearest code."""
    n = len(x)
    blocks = np.pad(np.abs(x), (0, -n % 256)).reshape(-1, 256).max(1)
    some = blocks > F(1e-30)
    scale = np.where(some, blocks * (F(1) / F(448)), F(0))
    per = np.repeat(np.where(some, F(1) / np.where(some, blocks, F(1)) * F(448), F(0)), 256)[:n]
    y = x * per
    a = np.abs(y)
    if u is not None:
        d = np.ldexp(F(1), np.maximum(np.frexp(a)[1] - 4, -9)).astype(F)
        a = np.floor(a / d + u) * d
    a = np.minimum(a, F(448))
    assert a.dtype == F and scale.dtype == F
    if root:
        a = np.where((x > 0) & (per > 0) & (a < F(2.0 ** -9)), F(2.0 ** -9), a)
    return torch.from_numpy(np.copysign(a, y)).to(torch.float8_e4m3fn), scale


@pytest.mark.parametrize("seeded", [False, True])
@pytest.mark.parametrize("g_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scaled", [False, True])
def test_codes_bit_by_bit(seeded, g_dtype, scaled):
    """Three steps over tensors of several sizes, one of them beyond a launch's forty."""
    tr = _train()
    rng = np.random.default_rng(3)
    sizes = [256, 1, 255, 1000, 0, 9000] + [70 + i for i in range(40)]
    plan = tr.AdamW("fp8")
    grads, ref = [], []
    for i, n in enumerate(sizes):
        grads.append(torch.zeros(n, device="cuda", dtype=g_dtype))
        plan.add(torch.zeros(n, device="cuda"), grads[-1])
        z = torch.zeros(n).to(torch.float8_e4m3fn)
        blocks = np.zeros(-(-n // 256), F)
        ref.append([z, blocks, z, blocks])
    factor = torch.tensor([0.37], device="cuda") if scaled else None
    beta, rest = [F(b) for b in BETAS], [F(1.0 - b) for b in BETAS]
    for t in range(1, 4):
        seed = 1000003 * t if seeded else 0
        for g, n in zip(grads, sizes):
            x = rng.standard_normal(n) * np.exp(2 * rng.standard_normal(n))
            x[:min(n, 300):7] = 0
            if n == 9000:
                x[512:768] = 0          # a block of zeros, and one below the least
                x[768:1024] *= 1e-34
            g.copy_(torch.from_numpy(x))
        plan.step(t, lr=1e-3, betas=BETAS, seed=seed, grad_scale=factor)
        torch.cuda.synchronize()
        for i, (g, r) in enumerate(zip(grads, ref)):
            x = g.float().cpu().numpy()
            if scaled:
                x = x * F(0.37)
            m = beta[0] * _values(r[0], r[1]) + rest[0] * x
            v = _values(r[2], r[3])
            v = beta[1] * (v * v) + (rest[1] * x) * x
            um, uv = _uniform(len(x), i, seed) if seeded else (None, None)
            r[:] = [*_code(m, um, False), *_code(np.sqrt(v), uv, True)]
            s = plan.kept[i]
            for name, want in zip(("m", "m_scale", "v", "v_scale"), r):
                got = s[name].cpu()
                if name in ("m", "v"):      # (a zero of either sign is zero)
                    assert torch.equal(got.float(), want.float()), (t, i, name)
                else:
                    assert np.array_equal(got.numpy(), want), (t, i, name)
