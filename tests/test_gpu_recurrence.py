"""The single-state recurrence and its backward pass against the recurrence itself in
float64, token by token, on the same inputs; and the calls it refuses.

Tolerances, relative to the reference's norm.  Products are summed in float32: a sum of n
terms of either sign is off by about sqrt(n) 2^-24 of its terms' size, and d_k + d_v + T
terms at most meet in an output: 1.5e-6 for the largest case here, of which ten times are
allowed for sums that cancel.  bfloat16: an output, the scores and the state that enter it
are each rounded once, by 2^-8 at most and less than half of that in the mean over
elements, so 2^-8 holds for the three together; states add up products whose factors keep
16 bits, 2^-16.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, STATE, BF16 = 1.5e-5, 2.0 ** -16, 2.0 ** -8
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _train():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import train
    return train


def make(B, H, Hk, T, dk, dv, dtype, *, state=True, lengths=None, g_lo=-0.05, cuts=0.0, layout="bthd",
         scale=1.0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(1000 + seed)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    dt = DT[dtype]

    def rows(heads, d, unit=False):
        x = rnd(B, T, heads, d)
        if unit:
            x = torch.nn.functional.normalize(x, dim=-1)
        if layout == "bthd":
            return x.to(dt).transpose(1, 2)
        if layout == "bhtd":
            return x.to(dt).transpose(1, 2).contiguous()
        wide = torch.full((B, T + 1, heads, d + 16), float("nan"), dtype=dt, device="cuda")   # a slice
        wide[:, :T, :, 8:8 + d] = x.to(dt)
        return wide[:, :T, :, 8:8 + d].transpose(1, 2)

    s = {"q": rows(Hk, dk, True), "k": rows(Hk, dk, True), "v": rows(H, dv), "do": rows(H, dv),
         "g": (g_lo * torch.rand((B, T, H), generator=gen, device="cuda")).transpose(1, 2),
         "S": rnd(B, H, dk, dv) / dk ** 0.5 if state else None,
         "dS": rnd(B, H, dk, dv) / dk ** 0.5 if state else None, "scale": scale, "len": None}
    if cuts:
        m = torch.rand((B, H, T), generator=gen, device="cuda")
        s["g"][m < cuts / 2] = float("-inf")
        s["g"][m > 1 - cuts / 2] = -200.0
    if lengths is not None:
        s["len"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        for b, n in enumerate(lengths):        # what lies behind the end counts for nothing
            n = max(n, 0)
            for name in ("q", "k", "v", "do", "g"):
                s[name][b, :, n:] = float("nan")
    return s


def reference(s, train=True):
    """float64, token by token: out, last state, dq, dk, dv, dg, gradient of the first state."""
    B, Hk, T, dk = s["q"].shape
    H, dv = s["v"].shape[1], s["v"].shape[3]
    n = s["len"].clamp(0, T).tolist() if s["len"] is not None else [T] * B
    live = torch.arange(T, device="cuda")[None] < torch.tensor(n, device="cuda")[:, None]
    f = lambda x: torch.where(live[:, None, :, None], x.double(), 0.0).repeat_interleave(H // x.shape[1], 1)  # noqa: E731
    q, k, v, do = f(s["q"]) * s["scale"], f(s["k"]), f(s["v"]), f(s["do"])
    g = torch.where(live[:, None], s["g"].double(), 0.0)
    a = torch.where(g < -87.33655, 0.0, g.exp())
    S = torch.zeros((B, H, dk, dv), dtype=torch.float64, device="cuda") if s["S"] is None else s["S"].double()
    out, states = [], []
    for t in range(T):
        states.append(S)
        S = S * a[:, :, t, None, None] + k[:, :, t, :, None] * v[:, :, t, None, :]
        out.append((S * q[:, :, t, :, None]).sum(2))
    r = {"out": torch.stack(out, 2), "state": S}
    if not train:
        return r
    R = torch.zeros_like(S) if s["dS"] is None else s["dS"].double()
    dq, dk_, dv_, dg = ([None] * T for _ in range(4))
    for t in reversed(range(T)):
        R = R + q[:, :, t, :, None] * do[:, :, t, None, :]
        now = states[t] * a[:, :, t, None, None]
        dq[t] = ((now + k[:, :, t, :, None] * v[:, :, t, None, :]) * do[:, :, t, None, :]).sum(3) * s["scale"]
        dk_[t] = (R * v[:, :, t, None, :]).sum(3)
        dv_[t] = (R * k[:, :, t, :, None]).sum(2)
        dg[t] = (R * now).sum((2, 3))
        R = R * a[:, :, t, None, None]
    group = lambda x: torch.stack(x, 2).unflatten(1, (Hk, H // Hk)).sum(2)  # noqa: E731
    r.update(dq=group(dq), dk=group(dk_), dv=torch.stack(dv_, 2), dg=torch.stack(dg, 2) * live[:, None], dstate=R)
    return r


def run(s, train=True, **kw):
    T_ = _train()
    args = dict(scale=s["scale"], state=s["S"], lengths=s["len"])
    out, last = T_.recurrence(s["q"], s["k"], s["v"], s["g"], want_state=True, **args, **kw)
    r = {"out": out, "state": last}
    if train:
        names = ("dq", "dk", "dv", "dg", "dstate")
        r.update(zip(names, T_.recurrence_backward(s["q"], s["k"], s["v"], s["g"], s["do"],
                                                   dstate=s["dS"], want_dstate=True, **args)))
    torch.cuda.synchronize()
    return r


def check(got, ref, bf16):
    for name, x in ref.items():
        y = got[name].double()
        tol = (STATE if name in ("state", "dstate") else BF16) if bf16 else F32
        assert torch.isfinite(y).all(), name
        err, norm = (y - x).norm().item(), x.norm().item()
        assert err <= tol * norm + 1e-30, (name, err / max(norm, 1e-30), tol)


SIZES = [(128, 128), (128, 64), (64, 128), (64, 64)]


@pytest.mark.parametrize("dk,dv", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 2, 6, 7, 12, 13, 31, 32, 33, 64, 97, 300])
def test_lengths_and_heads(T, dtype, dk, dv):
    s = make(2, 3, 3, T, dk, dv, dtype, seed=T)
    check(run(s), reference(s), dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk,dk,dv", [(6, 1, 128, 64), (6, 2, 64, 64), (4, 2, 128, 128), (3, 1, 64, 128)])
def test_shared_keys(H, Hk, dk, dv, dtype):
    s = make(2, H, Hk, 150, dk, dv, dtype, seed=H)
    check(run(s), reference(s), dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", [[0, 200, 77], [1, 32, 33], [199, -5, 1000], [0, 0, 0]])
def test_ragged(lengths, dtype):
    """Ends inside a chunk, at its edge, behind the tensor, and before the first token;
    NaN behind them in every input."""
    s = make(3, 2, 2, 200, 64, 128, dtype, lengths=lengths)
    got, ref = run(s), reference(s)
    check(got, ref, dtype == "bf16")
    for b, n in enumerate(lengths):
        n = min(max(n, 0), 200)
        for name in ("out", "dq", "dk", "dv", "dg"):
            assert not got[name][b, :, n:].any(), name
        if n == 0:
            assert torch.equal(got["state"][b], s["S"][b]) and torch.equal(got["dstate"][b], s["dS"][b])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_short_ragged(dtype):
    s = make(3, 2, 1, 5, 128, 64, dtype, lengths=[0, 5, 3])
    check(run(s), reference(s), dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cuts,g_lo", [(0.02, -0.05), (0.5, -0.05), (1.0, -0.05), (0.0, -20.0), (0.1, -80.0),
                                       (0.0, 0.0)])
def test_gates(cuts, g_lo, dtype):
    """Cut gates (-inf, and ones whose decay no normal float32 holds), steep ones, none.
    Beside a steep gate dg is small against the terms it is made of, and still right."""
    s = make(2, 2, 2, 260, 64, 64, dtype, cuts=cuts, g_lo=g_lo, state=cuts < 1)
    got, ref = run(s), reference(s)
    check(got, ref, dtype == "bf16")
    assert not got["dg"][s["g"] < -87.4].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["bhtd", "slice"])
def test_layouts(layout, dtype):
    s = make(2, 4, 2, 100, 128, 64, dtype, layout=layout)
    check(run(s), reference(s), dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_broadcast_inputs(dtype):
    """One key for all tokens, one gate for all heads (strides of zero)."""
    s = make(2, 3, 3, 80, 64, 64, dtype)
    s["k"] = s["k"][:, :, :1].expand(-1, -1, 80, -1)
    s["g"] = s["g"][:, :1].expand(-1, 3, -1)
    check(run(s), reference(s), dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.125, -2.0, 0.0])
def test_scale(scale, dtype):
    s = make(2, 2, 2, 130, 64, 64, dtype, scale=scale)
    check(run(s), reference(s), dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_states(dtype):
    s = make(2, 2, 2, 130, 128, 128, dtype, state=False)
    check(run(s), reference(s), dtype == "bf16")


@pytest.mark.parametrize("dtype,B,H,T", [("bf16", 1, 2, 2600), ("f32", 1, 1, 2600), ("bf16", 1, 300, 700),
                                         ("f32", 2, 130, 1100)])
def test_segments(dtype, B, H, T):
    """Few heads: sequences cut into segments, the last one short; many: one segment.  A
    ragged end and cut gates fall into the middle of segments."""
    s = make(B, H, H, T, 64, 64, dtype, cuts=0.002, lengths=[T - 333] * B)
    check(run(s), reference(s), dtype == "bf16")


def test_split_calls_continue():
    """T1 tokens, then T2 from the state they left, are T1 + T2 tokens."""
    tr = _train()
    s = make(1, 3, 3, 200, 128, 64, "f32")
    whole, last = tr.recurrence(s["q"], s["k"], s["v"], s["g"], state=s["S"], want_state=True)
    cut = lambda x, a, b: x[:, :, a:b]  # noqa: E731
    S = s["S"].clone()
    parts = []
    for a, b in ((0, 70), (70, 71), (71, 76), (76, 200)):
        o, S = tr.recurrence(*(cut(s[n], a, b) for n in ("q", "k", "v", "g")), state=S, state_out=S)
        parts.append(o)
    got = torch.cat(parts, 2)
    assert (got - whole).norm() <= F32 * whole.norm()
    assert (S - last).norm() <= F32 * last.norm()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_against_differences(dtype):
    """The gradients along random directions against central differences of the loss
    <out, do> + <state, dS>, evaluated in float64 from the definition."""
    s = make(1, 2, 1, 60, 64, 64, dtype)
    got = run(s)
    gen = torch.Generator(device="cuda").manual_seed(5)
    names = {"q": "dq", "k": "dk", "v": "dv", "g": "dg", "S": "dstate"}

    def loss(x):
        r = reference(x, train=False)
        return (r["out"] * s["do"].double()).sum() + (r["state"] * s["dS"].double()).sum()

    for name, grad in names.items():
        d = torch.randn(s[name].shape, generator=gen, device="cuda", dtype=torch.float64)
        eps = 1e-5
        up, down = dict(s), dict(s)
        up[name], down[name] = s[name].double() + eps * d, s[name].double() - eps * d
        want = ((loss(up) - loss(down)) / (2 * eps)).item()
        have = (got[grad].double() * d).sum().item()
        # a random direction meets the gradient's error at its norm's size
        size = got[grad].double().norm().item()
        tol = (STATE if grad == "dstate" else BF16) if dtype == "bf16" else F32
        assert abs(have - want) <= 4 * tol * size + 1e-6 * abs(want), (name, have, want)


def test_empty():
    tr = _train()
    s = make(2, 2, 2, 4, 64, 64, "bf16")
    z = {n: s[n][:, :, :0] for n in ("q", "k", "v", "g", "do")}
    out, last = tr.recurrence(z["q"], z["k"], z["v"], z["g"], state=s["S"], want_state=True)
    assert out.shape == (2, 2, 0, 64) and torch.equal(last, s["S"])
    _, last = tr.recurrence(z["q"], z["k"], z["v"], z["g"], want_state=True)
    assert not last.any()
    g = tr.recurrence_backward(z["q"], z["k"], z["v"], z["g"], z["do"], state=s["S"], dstate=s["dS"])
    assert torch.equal(g[4], s["dS"])
    z = {n: s[n][:0] for n in ("q", "k", "v", "g")}
    assert tr.recurrence(z["q"], z["k"], z["v"], z["g"])[0].shape == (0, 2, 4, 64)


@pytest.mark.parametrize("T", [3, 150])
def test_in_place_and_repeatable(T):
    """The state updated in place, the gradient of a state over the incoming one, and the
    same bits from call to call, on a side stream too."""
    tr = _train()
    s = make(1, 4, 2, T, 64, 128, "bf16")
    first = run(s)
    S = s["S"].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out, last = tr.recurrence(s["q"], s["k"], s["v"], s["g"], state=S, state_out=S)
        again = tr.recurrence_backward(s["q"], s["k"], s["v"], s["g"], s["do"], state=s["S"], dstate=s["dS"])
    torch.cuda.synchronize()
    assert last is S and torch.equal(out, first["out"]) and torch.equal(S, first["state"])
    for name, x in zip(("dq", "dk", "dv", "dg", "dstate"), again):
        assert torch.equal(x, first[name]), name


def test_graph():
    """Forward and backward in a recorded graph, replayed over new inputs, with eager work
    between the replays."""
    tr = _train()
    s = make(1, 4, 4, 700, 64, 64, "bf16")
    ws = torch.empty(tr.recurrence_workspace_bytes(1, 4, 4, 700, 64, 64, torch.bfloat16, backward=True),
                     dtype=torch.uint8, device="cuda")
    call = lambda: (tr.recurrence(s["q"], s["k"], s["v"], s["g"], state=s["S"], want_state=True, workspace=ws) +  # noqa: E731
                    tr.recurrence_backward(s["q"], s["k"], s["v"], s["g"], s["do"], state=s["S"],
                                           dstate=s["dS"], workspace=ws))
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for i in range(3):
        new = make(1, 4, 4, 700, 64, 64, "bf16", seed=50 + i)
        for n in ("q", "k", "v", "g", "do", "S", "dS"):
            s[n].copy_(new[n])
        graph.replay()
        torch.cuda.synchronize()
        kept = [x.clone() for x in got]
        for x, y in zip(kept, call()):
            assert torch.equal(x, y)
        torch.cuda.synchronize()


def test_refusals():
    """Arguments the entry points refuse, by status and before any work."""
    tr = _train()
    from paper_2606_10650_amd import dla
    s = make(1, 2, 2, 40, 64, 64, "bf16")
    q, k, v, g = s["q"], s["k"], s["v"], s["g"]

    def status(f, want):
        with pytest.raises(dla.DLAError) as e:
            f()
        assert e.value.status == want

    x = torch.zeros((1, 2, 40, 96), dtype=torch.bfloat16, device="cuda")
    status(lambda: tr.recurrence(x, x, v, g), dla.DLA_ERR_UNSUPPORTED)                 # d_k 96
    three = torch.zeros((1, 3, 40, 64), dtype=torch.bfloat16, device="cuda")
    status(lambda: tr.recurrence(q, k, three, torch.zeros((1, 3, 40), device="cuda")),
           dla.DLA_ERR_INVALID_ARG)                                                     # 3 heads, 2 key heads
    odd = torch.zeros(40 * 2 * 65 + 8, dtype=torch.bfloat16, device="cuda")
    skew = odd.as_strided((1, 2, 40, 64), (0, 65, 130, 1))
    status(lambda: tr.recurrence(skew, k, v, g), dla.DLA_ERR_INVALID_ARG)              # rows of 130 bytes
    status(lambda: tr.recurrence(q, k, odd[1:].as_strided((1, 2, 40, 64), (0, 64, 128, 1)), g),
           dla.DLA_ERR_INVALID_ARG)                                                     # base off by 2 bytes
    status(lambda: tr.recurrence(q, k, v, g, out=torch.zeros_like(v)[:, :, :1].expand(-1, -1, 40, -1)),
           dla.DLA_ERR_INVALID_ARG)                                                     # overlapping outputs
    with pytest.raises(ValueError):
        tr.recurrence(q, k, v, g.bfloat16())
    with pytest.raises(ValueError):
        tr.recurrence(q, k.float(), v, g)
    with pytest.raises(ValueError):
        tr.recurrence(q, k, v, g, state=torch.zeros((1, 2, 64, 32), device="cuda"))
    with pytest.raises(ValueError):
        tr.recurrence(q, k, v, g, lengths=torch.zeros(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        tr.recurrence(q, k, v.transpose(2, 3).contiguous().transpose(2, 3), g)          # last axis strided
    # a short or unaligned workspace
    L = tr.lib()
    out = torch.empty_like(v)
    args = [tr._desc(1, 2, 2, 40, 64, 64, torch.bfloat16), tr._rows(q, "q"), tr._rows(k, "k"), tr._rows(v, "v"),
            tr._rows(g, "g"), None, tr._rows(out, "out"), None]
    need = tr.recurrence_workspace_bytes(1, 2, 2, 40, 64, 64, torch.bfloat16)
    ws = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    for p, n in ((None, need), (ws.data_ptr(), need - 1), (ws.data_ptr() + 64, need)):
        assert L.dla_recurrence_forward(*args, p, n, None) == dla.DLA_ERR_WORKSPACE
