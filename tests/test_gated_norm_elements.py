"""The gated norm's outputs and gradients element by element, with row means that count, and, without a GPU, that the
bounds reject what a kernel could get wrong: a mean left out, a tail left out, a row missing from a weight's gradient.

Bounds.  U = 2^-24 is float32's half step.  A sum over a row goes through at most 32 values of a thread, 6 steps of a
wave and 15 of a workgroup: DEPTH = 56 with the rounding of the terms, of one sign for a sum of squares, so that 1 / sqrt
of it is off by ER = (DEPTH / 2 + 7) U of itself.  A sigmoid s(z) is off by ES = (5 + 1.3 |z| (1 - s)) U of itself: an
exponential whose argument is rounded, a sum, a reciprocal.  Errors of factors add, those of summands are summed
as magnitudes, and each operation adds U of its result: `bounds` follows the formulas line by line.  What is stored is
rounded once, by half a step of its type, 2^-8 or U of the value."""
import pytest
import torch

U = 2.0 ** -24
DEPTH = 56
ER = (DEPTH / 2 + 7) * U
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": U}
EPS = 1e-5
FORMS = [dict(), dict(gate=True), dict(residual=True, scale=0.5), dict(gate=True, residual=True, next=True, scale=0.25),
         dict(residual=True, next=True), dict(next=True, gate=True)]
ROWS = [(1, 1), (3, 2), (5, 7), (4, 64), (33, 65), (7, 512), (4, 1000), (300, 1531), (260, 2048), (9, 2049), (5, 4100), (3, 8200), (2, 16384)]
GROUPS = [(4, 2, 1), (4, 3, 64), (50, 16, 128), (9, 48, 64), (700, 5, 40), (3, 33, 300), (3, 7, 1000), (2, 2, 5000), (3, 5, 2200)]


def make(N, G, D, dtype, *, gate=False, residual=False, next=False, scale=1.0, per_group=False, wf32=False, device="cpu"):  # noqa: A002
    """Gradients that go along with what they are gradients of, so that the rows' means are of order one."""
    gen = torch.Generator().manual_seed(11 + 7 * N + 3 * G + D)
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    dt = DT[dtype]
    wdt = torch.float32 if wf32 else dt
    row = lambda t: t.to(dt)  # noqa: E731
    s = dict(x=row(torch.exp(2 * rnd(N, G, 1)) * rnd(N, G, D)), gate=row(2 * rnd(N, G, D)) if gate else None,
             residual=row(rnd(N, G, D)) if residual else None, w=(1 + 0.2 * (rnd(G, D) if per_group else rnd(D))).to(wdt),
             next=(1 + 0.2 * rnd(D)).to(wdt) if next else None, scale=scale)
    s["dh"], s["dy"] = row(rnd(N, G, D)), row(rnd(N, G, D)) if next else None
    v = values(s)
    s["dh"] = row(s["dh"].double() + v["n"] * v["act"])
    if next:
        s["dy"] = row(s["dy"].double() + v["n2"])
    return {k: t.to(device) if torch.is_tensor(t) else t for k, t in s.items()}


def values(s, without=()):
    """Everything in float64; `without`: means taken as zero, for results that must be told from the right ones."""
    d = lambda k: None if s[k] is None else s[k].double()  # noqa: E731
    x, z, res, w, w2, dh, dy, k = d("x"), d("gate"), d("residual"), d("w"), d("next"), d("dh"), d("dy"), s["scale"]
    v = dict(r=1 / (x.square().mean(-1, keepdim=True) + EPS).sqrt())
    v["n"] = n = x * v["r"]
    v["s"] = q = None if z is None else torch.sigmoid(z)
    v["act"] = act = torch.ones_like(x) if z is None else z * q
    v["b"] = n * w * act
    v["h"] = h = k * v["b"] + (0 if res is None else res)
    v["into"] = dh
    if w2 is not None:
        v["r2"] = 1 / (h.square().mean(-1, keepdim=True) + EPS).sqrt()
        v["n2"] = h * v["r2"]
        v["y"] = v["n2"] * w2
        v["m2"] = (dy * w2 * v["n2"]).mean(-1, keepdim=True) * (0 if "m2" in without else 1)
        v["into"] = dh + v["r2"] * (dy * w2 - v["n2"] * v["m2"])
        v["dnext"] = (dy * v["n2"]).sum((0, 1))
    v["db"] = db = k * v["into"]
    if z is not None:
        v["slope"] = q * (1 + z * (1 - q))
        v["dgate"] = db * n * w * v["slope"]
    v["d"] = db * act * w
    v["m"] = (v["d"] * n).mean(-1, keepdim=True) * (0 if "m" in without else 1)
    v["dx"] = v["r"] * (v["d"] - n * v["m"])
    each = db * act * n
    v["dw"] = each.sum(0) if w.dim() == 2 else each.sum((0, 1))
    return v


def bounds(s, v):
    """How far float32's results may be from v before they are stored."""
    a = lambda t: t.abs()  # noqa: E731
    over = lambda t: t.sum(0) if s["w"].dim() == 2 else t.sum((0, 1))  # noqa: E731
    D, N, k, w, n = s["x"].shape[-1], s["x"].shape[0], abs(s["scale"]), s["w"].double().abs(), v["n"].abs()
    e, es, eslope = {}, 0.0, 0.0
    if v["s"] is not None:
        z, q = s["gate"].double(), v["s"]
        es = (5 + 1.3 * a(z) * (1 - q)) * U
        eslope = q * (es * a(1 + z * (1 - q)) + a(z) * (q * es + U) + 3 * U * (1 + a(z) * (1 - q)))
    e["h"] = a(k * v["b"]) * (ER + 6 * U + es) + U * a(v["h"])
    into = e2 = 0.0
    if s["next"] is not None:
        w2, dy, n2, r2, m2 = s["next"].double().abs(), a(s["dy"].double()), a(v["n2"]), v["r2"], a(v["m2"])
        er2 = e["h"].norm(dim=-1, keepdim=True) / v["h"].norm(dim=-1, keepdim=True) + ER
        e2 = r2 * e["h"] + n2 * (er2 + U)
        e["y"] = w2 * e2 + U * a(v["y"])
        em = (dy * w2 * e2).mean(-1, keepdim=True) + DEPTH * U * (dy * w2 * n2).mean(-1, keepdim=True) + U * m2
        into = r2 * (e2 * m2 + n2 * em + (3 * U + er2) * (dy * w2 + n2 * m2)) + U * a(v["into"])
        e["dnext"] = (dy * e2).sum((0, 1)) + (N + 40) * U * (dy * n2).sum((0, 1))
    e["dres"] = into + 0 * n
    edb = k * into + U * a(v["db"])
    if v["s"] is not None:
        e["dgate"] = edb * n * w * a(v["slope"]) + a(v["dgate"]) * (ER + 5 * U) + a(v["db"]) * n * w * eslope
    ed = edb * a(v["act"]) * w + a(v["d"]) * (es + 4 * U)
    em = (ed * n + a(v["d"]) * n * (ER + U)).mean(-1, keepdim=True) + DEPTH * U * (a(v["d"]) * n).mean(-1, keepdim=True) + U * a(v["m"])
    e["dx"] = v["r"] * (ed + n * em + (ER + 2 * U) * n * a(v["m"]) + 2 * U * (a(v["d"]) + n * a(v["m"]))) + (ER + U) * a(v["dx"])
    each = edb * a(v["act"]) * n + a(v["db"] * v["act"]) * n * (ER + es + 3 * U)
    e["dw"] = over(each) + (N + 40) * U * over(a(v["db"] * v["act"]) * n)
    return e


def wanted(s):
    """(names of a call's outputs, their values, their bounds)"""
    v = values(s)
    v["dres"] = v["into"]
    names = ["h", "dx", "dw"] + ["dgate"] * (s["gate"] is not None) + ["dres"] * (s["residual"] is not None) + ["y", "dnext"] * (s["next"] is not None)
    return names, v, bounds(s, v)


def wrong(got, names, v, e, half):
    """The outputs of which some element is further off than its bound."""
    bad = []
    for name in names:
        own = U if name in ("dw", "dnext") else half
        g = got[name].double()
        off = own * v[name].abs() + (1 + own) * e[name] + 2.0 ** -126
        if not torch.isfinite(g).all() or not ((g - v[name]).abs() <= off).all():
            bad.append(name)
    return bad


def stored(names, v, dtype):
    return {k: v[k].to(torch.float32 if k in ("dw", "dnext") else DT[dtype]) for k in names}


CASES = [(N, 1, D, dict(form, wf32=i % 2 == 1)) for N, D in ROWS for i, form in enumerate(FORMS)]
CASES += [(N, G, D, dict(form, per_group=per)) for N, G, D in GROUPS for form in FORMS[:3] for per in (False, True)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,G,D", sorted({c[:3] for c in CASES}))
def test_bounds_tell(N, G, D, dtype):
    """The right results, rounded, are taken; those of which something is left out are not."""
    for _, _, _, form in (c for c in CASES if c[:3] == (N, G, D)):
        s = make(N, G, D, dtype, **form)
        names, v, e = wanted(s)
        right = stored(names, v, dtype)
        tell = lambda **kw: wrong({**right, **kw}, names, v, e, HALF[dtype])  # noqa: E731
        assert tell() == []
        cast = lambda t: t.to(DT[dtype])  # noqa: E731
        if D > 1:        # (a row of one value is its own mean)
            assert tell(dx=cast(values(s, ("m",))["dx"])) == ["dx"], form
        if s["next"] is not None:
            less = values(s, ("m2",))
            assert "dx" in tell(dx=cast(less["dx"])) or D == 1, form
            if s["residual"] is not None:
                assert tell(dres=cast(less["into"])) == ["dres"], form
        for name in names:
            if name in ("dw", "dnext"):
                continue
            for tail in (1, 8):
                t = right[name].clone()
                t[..., -tail:] = 0
                # (of a row of one value dx is next to nothing)
                assert tell(**{name: t}) == [name] or (D == 1 and name == "dx"), (form, name, tail)
        if N > 1:        # the last row missing from the weights' gradients
            less = values({k: t[:-1] if torch.is_tensor(t) and k not in ("w", "next") else t for k, t in s.items()})
            for name in ("dw", "dnext"):
                if name in names:
                    assert tell(**{name: less[name].float()}) == [name], (form, name)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,G,D", sorted({c[:3] for c in CASES}))
def test_elements(N, G, D, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import block
    for _, _, _, form in (c for c in CASES if c[:3] == (N, G, D)):
        s = make(N, G, D, dtype, device="cuda", **form)
        h, y, rstd, y_rstd = block.gated_norm(s["x"], s["w"], s["gate"], s["residual"], scale=s["scale"], next_weight=s["next"], eps=EPS)
        g = block.gated_norm_backward(s["dh"], s["x"], s["w"], rstd, s["gate"], s["residual"], scale=s["scale"], next_weight=s["next"],
                                      dy=s["dy"], y_rstd=y_rstd)
        got = dict(zip(("dx", "dgate", "dres", "dw", "dnext"), g), h=h, y=y)
        names, v, e = wanted(s)
        assert wrong(got, names, v, e, HALF[dtype]) == [], form
