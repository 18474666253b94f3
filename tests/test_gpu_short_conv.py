"""The short causal convolution and its backward pass against their formulas in float64, token by
token; states carried from call to call, documents, ragged ends, strides; and what is refused.

Tolerances, element by element.  z is a float32 sum of at most W + 1 terms, each product rounded
once: off by at most (2 W + 2) 2^-24 of the sum S of the terms' magnitudes.  The sigmoid is off by
at most (8 + 2 |z|) 2^-24 of itself (an exponential of a rounded multiple of z, a sum, a
reciprocal), silu and its slope by as much and by what z is off (|silu'| < 1.1, |silu''| <= 0.5).
Outputs in bfloat16 are rounded once more, by 2^-8 of their value.  dweight's sums are of n terms:
n 2^-24 of the magnitudes at most, and what their terms are off.
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


def make(B, T, C, W, dtype, *, bias=False, state=False, lengths=False, starts=0.0, wf32=False, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + 31 * T + C)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    dt = DT[dtype]
    wdt = torch.float32 if wf32 else dt
    s = {"x": rnd(B, T, C).to(dt), "w": rnd(C, W).to(wdt), "bias": rnd(C).to(wdt) if bias else None,
         "S": rnd(B, W - 1, C).to(dt) if state else None, "dy": rnd(B, T, C).to(dt),
         "dS": rnd(B, W - 1, C).to(dt), "len": None, "starts": None}
    if lengths:
        n = torch.randint(-2, T + 3, (B,), generator=gen, device="cuda", dtype=torch.int32)
        n[0] = min(1, T)
        s["len"] = n
        behind = torch.arange(T, device="cuda")[None] >= n[:, None]
        s["x"][behind] = float("nan")
        s["dy"][behind] = float("nan")
    if starts:
        s["starts"] = torch.rand((B, T), generator=gen, device="cuda") < starts
    return s


def oracle(s, silu):
    """out, state, dx, dw, dbias, dstate in float64, and bounds of what each may be off before rounding."""
    x, w = s["x"].double().cpu(), s["w"].double().cpu()
    B, T, C = x.shape
    W = w.shape[1]
    z64 = lambda *sh: torch.zeros(sh, dtype=torch.float64)  # noqa: E731
    bias = z64(C) if s["bias"] is None else s["bias"].double().cpu()
    S = z64(B, W - 1, C) if s["S"] is None else s["S"].double().cpu()
    dy, dS = s["dy"].double().cpu(), s["dS"].double().cpu()
    n = [T] * B if s["len"] is None else [min(max(int(v), 0), T) for v in s["len"]]
    starts = torch.zeros((B, T), dtype=torch.bool) if s["starts"] is None else s["starts"].cpu()
    r = {k: z64(B, T, C) for k in ("out", "dx", "out_off", "dx_off")}
    r.update(state=z64(B, W - 1, C), dstate=z64(B, W - 1, C), dstate_off=z64(B, W - 1, C), dw=z64(C, W),
             dw_off=z64(C, W), dbias=z64(C), dbias_off=z64(C))
    for b in range(B):
        seq = torch.cat([S[b], x[b, :n[b]]])                    # row i is token i - (W - 1)
        d, off = torch.zeros_like(seq), torch.zeros_like(seq)
        first = 0                                               # of the document, as a row of seq
        for t in range(n[b]):
            if starts[b, t]:
                first = t + W - 1
            rows = [i for i in range(t, t + W) if i >= first]
            z, mag = bias.clone(), bias.abs()
            for i in rows:
                z += w[:, i - t] * seq[i]
                mag = mag + (w[:, i - t] * seq[i]).abs()
            dz_ = (2 * W + 2) * U * mag
            q = torch.sigmoid(z) if silu else torch.ones(C, dtype=torch.float64)
            slope = q * (1 + z * (1 - q)) if silu else q
            r["out"][b, t] = z * q
            r["out_off"][b, t] = 1.1 * dz_ + (10 + 2 * z.abs()) * U * (z * q).abs()
            g = dy[b, t] * slope
            goff = dy[b, t].abs() * (0.5 * dz_ + (16 + 4 * z.abs()) * U) if silu else torch.zeros(C, dtype=torch.float64)
            for i in rows:
                d[i] += w[:, i - t] * g
                off[i] += w[:, i - t].abs() * (goff + 2 * W * U * g.abs())
                r["dw"][:, i - t] += g * seq[i]
                r["dw_off"][:, i - t] += (goff + (B * T + 8) * U * g.abs()) * seq[i].abs()
            r["dbias"] += g
            r["dbias_off"] += goff + (B * T + 8) * U * g.abs()
        for j in range(W - 1):
            i = n[b] + j
            if i >= first:
                r["state"][b, j] = seq[i]
                d[i] += dS[b, j]
                off[i] += 2 * W * U * dS[b, j].abs()
        r["out"][b, t + 1 if n[b] else 0:] = 0
        r["dx"][b, :n[b]], r["dx_off"][b, :n[b]] = d[W - 1:], off[W - 1:]
        r["dstate"][b], r["dstate_off"][b] = d[:W - 1], off[:W - 1]
    return r


def close(got, want, off, half):
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    # (what is below the smallest normal number may be zero)
    bad = (got - want).abs() > off + (half * 1.001) * (want.abs() + off) + 2.0 ** -126
    assert not bad.any(), ((got - want).abs() / (off + half * want.abs() + 1e-37)).max()


def run(block, s, silu, **kw):
    act = "silu" if silu else None
    common = dict(activation=act, state=s["S"], lengths=s["len"], starts=s["starts"])
    out, last = block.short_conv(s["x"], s["w"], s["bias"], want_state=True, **common)
    dx, dw, db, ds = block.short_conv_backward(s["x"], s["w"], s["dy"], s["bias"], dstate=s["dS"], want_dstate=True,
                                               **common)
    return {"out": out, "state": last, "dx": dx, "dw": dw, "dbias": db, "dstate": ds}


def check(got, s, silu, dtype):
    r = oracle(s, silu)
    close(got["out"], r["out"], r["out_off"], HALF[dtype])
    assert torch.equal(got["state"].double().cpu(), r["state"])
    close(got["dx"], r["dx"], r["dx_off"], HALF[dtype])
    close(got["dstate"], r["dstate"], r["dstate_off"], HALF[dtype])
    close(got["dw"], r["dw"], r["dw_off"], U)
    if s["bias"] is not None:
        close(got["dbias"], r["dbias"], r["dbias_off"], U)


@pytest.mark.parametrize("B,T,C,W", [(1, 1, 1, 2), (2, 1, 64, 4), (3, 2, 7, 4), (1, 3, 8, 4), (2, 9, 65, 3), (1, 64, 24, 2),
                                     (2, 77, 130, 4), (5, 40, 3, 3), (1, 300, 72, 4)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("silu", [True, False])
def test_forward_and_backward(B, T, C, W, dtype, silu):
    block = _block()
    for opt in (dict(), dict(bias=True, state=True, starts=0.2), dict(state=True, lengths=True, wf32=True),
                dict(lengths=True, starts=0.5, bias=True)):
        s = make(B, T, C, W, dtype, **opt)
        check(run(block, s, silu), s, silu, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_runs(dtype):
    """Sequences that many threads walk along, each its run, and many sequences for few threads."""
    block = _block()
    for B, T, C in ((1, 4000, 16), (700, 5, 9)):
        s = make(B, T, C, 4, dtype, state=True, starts=0.05, lengths=B > 1)
        check(run(block, s, True), s, True, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_runs_than_workgroups(dtype):
    """So many sequences that a workgroup of the backward pass takes several; without a state or documents the
    formula is a sum over shifted arrays."""
    block = _block()
    B, T, C, W = 300000, 2, 8, 3
    s = make(B, T, C, W, dtype)
    out, _ = block.short_conv(s["x"], s["w"], activation=None)
    dx, dw, _, _ = block.short_conv_backward(s["x"], s["w"], s["dy"], activation=None)
    x, w, dy = (s[k].double() for k in ("x", "w", "dy"))
    off = lambda mag: 2 * W * U * mag + HALF[dtype] * 1.001 * mag + 2.0 ** -126  # noqa: E731
    z = x * w[:, 2] + torch.nn.functional.pad(x, (0, 0, 1, 0))[:, :T] * w[:, 1]
    mag = (x * w[:, 2]).abs() + (torch.nn.functional.pad(x, (0, 0, 1, 0))[:, :T] * w[:, 1]).abs()
    assert ((out.double() - z).abs() <= off(mag)).all()
    next_ = torch.nn.functional.pad(dy, (0, 0, 0, 1))[:, 1:]
    assert ((dx.double() - dy * w[:, 2] - next_ * w[:, 1]).abs() <= off((dy * w[:, 2]).abs() + (next_ * w[:, 1]).abs())).all()
    want = torch.stack([torch.zeros(C, dtype=torch.float64, device="cuda"), (dy[:, 1] * x[:, 0]).sum(0), (dy * x).sum((0, 1))], 1)
    # a thread adds up few terms in float32, the rest is float64: 64 2^-24 of the terms' magnitudes
    assert ((dw.double() - want).abs() <= 64 * U * (dy.abs().sum((0, 1)) * x.abs().max())[:, None]).all()


def test_strides_and_slices():
    """Slices of a wider projection at any element, transposed and broadcast sequences."""
    block = _block()
    for off, C in ((0, 24), (1, 24), (8, 13)):
        s = make(2, 21, C, 4, "bf16", starts=0.2)
        plain = run(block, s, True)
        for wide in (40, 41):
            x, dy = (torch.full((21, 2, wide), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            for a, k in ((x, "x"), (dy, "dy")):
                a[..., off:off + C] = s[k].transpose(0, 1)
            v = dict(s, x=x[..., off:off + C].transpose(0, 1), dy=dy[..., off:off + C].transpose(0, 1))
            got = run(block, v, True)
            for k in plain:
                if plain[k] is not None:
                    assert torch.equal(plain[k], got[k]), k
            out = torch.full((2, 21, wide), 7.0, dtype=torch.bfloat16, device="cuda")
            block.short_conv(v["x"], s["w"], starts=s["starts"], out=out[..., off:off + C])
            assert torch.equal(out[..., off:off + C], plain["out"])
            assert (out[..., :off] == 7).all() and (out[..., off + C:] == 7).all()
    one = make(1, 21, 24, 3, "f32")
    many = dict(one, x=one["x"].expand(3, -1, -1), dy=one["dy"].expand(3, -1, -1), dS=one["dS"].repeat(3, 1, 1))
    a, b = run(block, one, True), run(block, many, True)
    assert torch.equal(b["out"], a["out"].expand(3, -1, -1)) and torch.equal(b["dx"], a["dx"].expand(3, -1, -1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_state_carries_on(dtype):
    """A sequence in parts, the state passed in place, gives what it gives at once, bit by bit."""
    block = _block()
    s = make(3, 50, 40, 4, dtype, state=True, starts=0.1)
    whole, last = block.short_conv(s["x"], s["w"], state=s["S"], starts=s["starts"], want_state=True)
    state, outs, at = s["S"].clone(), [], 0
    for n in (1, 1, 2, 1, 0, 20, 3, 22):
        o, back = block.short_conv(s["x"][:, at:at + n], s["w"], state=state, state_out=state,
                                   starts=s["starts"][:, at:at + n].contiguous())
        assert back is state
        outs.append(o)
        at += n
    assert torch.equal(torch.cat(outs, 1), whole) and torch.equal(state, last)


def test_gradient_against_differences():
    """dx, dw, dbias and dstate against central differences of the float32 call: of a loss L that is a
    sum of n outputs, each off by some 2^-22, the difference over 2 h is off by n 2^-22 / 2 h, and by
    h^2 / 6 of a third derivative of order one."""
    block = _block()
    s = make(2, 12, 5, 3, "f32", bias=True, state=True, starts=0.2)
    names = (("x", "dx"), ("w", "dw"), ("bias", "dbias"), ("S", "dstate"))
    g = run(block, s, True)
    loss = lambda v: sum((a.double() * b.double()).sum() for a, b in zip(  # noqa: E731
        block.short_conv(v["x"], v["w"], v["bias"], state=v["S"], starts=v["starts"], want_state=True),
        (s["dy"], s["dS"])))
    gen, h = torch.Generator(device="cuda").manual_seed(5), 2.0 ** -6
    for name, grad in names:
        for _ in range(3):
            d = torch.randn(s[name].shape, generator=gen, device="cuda")
            d /= d.norm()
            num = (loss(dict(s, **{name: s[name] + h * d})) - loss(dict(s, **{name: s[name] - h * d}))) / (2 * h)
            # (120 outputs of order one: 120 2^-22 2^5 = 1e-3; h^2 = 2.4e-4 times derivatives of up to 10)
            assert abs((g[grad].double() * d.double()).sum() - num) < 5e-3


def test_same_bits_again_and_on_another_stream():
    block = _block()
    s = make(4, 333, 200, 4, "bf16", state=True, starts=0.1, lengths=True, bias=True)
    a = run(block, s, True)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        b = run(block, s, True)
    stream.synchronize()
    for k in a:
        assert torch.equal(a[k], b[k]), k


def test_captured():
    """A step in a graph, replayed over new inputs with the state in place, with eager calls between."""
    block = _block()
    s = make(8, 1, 96, 4, "bf16", state=True)
    x, state = s["x"].clone(), s["S"].clone()
    out = torch.empty_like(x)
    block.short_conv(x, s["w"], state=state, state_out=state, out=out)
    state.copy_(s["S"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.short_conv(x, s["w"], state=state, state_out=state, out=out)
    state.copy_(s["S"])
    ref = s["S"].clone()
    for i in range(5):
        x.copy_(torch.randn(x.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i)))
        want, _ = block.short_conv(x, s["w"], state=ref, state_out=ref)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(state, ref)


def test_empty():
    block = _block()
    for B, T, C in ((0, 5, 8), (2, 0, 8), (2, 5, 0)):
        s = make(B, T, C, 4, "f32", state=True)
        got = run(block, s, True)
        if T == 0:
            assert torch.equal(got["state"], s["S"]) and torch.equal(got["dstate"], s["dS"])
        assert not got["dw"].any()
