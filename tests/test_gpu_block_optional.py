"""Outputs that a caller of dla_block.h may leave out, and gradients that may be NULL for zero, each in turn: what is left
has the bits of the whole call, whatever the workspace held."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
NAN = float("nan")


def _block():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10650_amd import block
    return block


def _rnd(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(s, generator=gen, device="cuda")


def _ws(n):
    """n bytes, all ones: NaN as bfloat16 and as float32."""
    return torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda")


def _same(got, want, names):
    for k in names:
        assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,F", [(5, 16, 24), (70, 40, 72), (100, 33, 51), (300, 104, 40), (700, 328, 520), (4100, 520, 1544)])
def test_feed_forward(N, D, F, dtype):
    """One half of the weights' product alone, where a tile holds the end of one half and the start of the other (F is no
    multiple of 32); without dx the weights are not packed."""
    block, rnd, dt = _block(), _rnd(N), DT[dtype]
    x, wg, wu, dy = (t.to(dt) for t in (rnd(N, D), rnd(F, D) / D ** 0.5, rnd(F, D) / D ** 0.5, rnd(N, F)))
    y, parts = block.gated_ff(x, wg, wu, want_parts=True)
    assert torch.equal(block.gated_ff(x, wg, wu)[0], y)
    want = dict(zip(("dx", "dwg", "dwu"), block.gated_ff_backward(x, wg, wu, parts, dy)))
    desc = block._FF.pack(N, D, F, block._code(dt))
    row = lambda t: block._ROWS.pack(t.data_ptr(), t.stride(0))  # noqa: E731
    for names in (("dwg", "dwu"), ("dx",), ("dx", "dwg"), ("dx", "dwu"), ("dwg",), ("dwu",), ()):
        got = {k: torch.full_like(want[k], NAN) for k in names}
        ws = _ws(block.gated_ff_workspace_bytes(N, D, F, dt, backward=True, aligned=block._aligned(x, wg, wu)))
        block._call("dla_gated_ff_backward", x.device, desc, row(x), row(wg), row(wu), row(parts[0]), row(parts[1]), row(dy),
                    *(row(got[k]) if k in got else None for k in ("dx", "dwg", "dwu")), ws.data_ptr(), ws.numel())
        _same(got, want, names)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,G,D", [(40, 1, 64), (7, 1, 700), (300, 1, 2048), (5, 1, 9000), (30, 6, 48)])
def test_gated_norm(N, G, D, dtype):
    block, rnd, dt = _block(), _rnd(D), DT[dtype]
    x, gate, res, dh, dy = (rnd(N, G, D).to(dt) for _ in range(5))
    w, w2 = (1 + 0.2 * rnd(D)).to(dt), (1 + 0.2 * rnd(D)).to(dt) if G == 1 else None
    dy = dy if G == 1 else None
    h, y, rstd, y_rstd = block.gated_norm(x, w, gate, res, scale=0.5, next_weight=w2)
    desc = block._gated_desc(x, w, w2, 1e-6, 0.5)
    row = lambda t: None if t is None else block._group_rows(t, x, "t")  # noqa: E731
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    # statistics that nobody wants
    for skip in ((), ("rstd",), ("y_rstd",), ("rstd", "y_rstd")):
        got = {"h": torch.full_like(x, NAN), "y": torch.full_like(x, NAN) if G == 1 else None, "rstd": torch.full_like(rstd, NAN),
               "y_rstd": None if y_rstd is None else torch.full_like(y_rstd, NAN)}
        block._call("dla_gated_norm", x.device, desc, row(x), row(gate), row(res), w.data_ptr(), ptr(w2), row(got["h"]), row(got["y"]),
                    *(None if k in skip else ptr(got[k]) for k in ("rstd", "y_rstd")))
        _same(got, dict(h=h, y=y, rstd=rstd, y_rstd=y_rstd), [k for k in got if got[k] is not None and k not in skip])
    shapes = dict(dx=x, dgate=x, dres=x, dw=torch.empty(D, device="cuda"), dw2=torch.empty(D, device="cuda"))

    def back(left, dh, dy, space=True):
        got = {k: torch.full_like(t, NAN) for k, t in shapes.items() if k not in left and (k != "dw2" or G == 1)}
        ws = _ws(block.gated_norm_workspace_bytes(N, G, D, dt))
        block._call("dla_gated_norm_backward", x.device, desc, row(x), row(gate), row(res), w.data_ptr(), ptr(w2), rstd.data_ptr(),
                    ptr(y_rstd), row(dh), row(dy), row(got["dx"]), *(row(got.get(k)) for k in ("dgate", "dres")),
                    *(ptr(got.get(k)) for k in ("dw", "dw2")), ws.data_ptr() if space else None, ws.numel() if space else 0)
        return got

    for grads in ((dh, dy), (dh, None), (None, dy)):
        want = back((), *grads)
        for t in want.values():
            assert torch.isfinite(t).all()
        for left in (("dgate",), ("dres",), ("dw",), ("dw2",), ("dgate", "dres"), ("dw", "dw2"), ("dgate", "dres", "dw", "dw2")):
            got = back(left, *grads, space="dw" not in left or "dw2" not in left)
            _same(got, want, got)
    zero = back((), torch.zeros_like(dh), dy)
    _same(back((), None, dy), zero, zero)
    if dy is not None:
        zero = back((), dh, torch.zeros_like(dy))
        _same(back((), dh, None), zero, zero)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,C", [(3, 1, 40), (2, 70, 33), (2, 400, 136)])
def test_short_conv(B, T, C, dtype):
    block, rnd, dt = _block(), _rnd(T), DT[dtype]
    x, dy, S, dS = (t.to(dt) for t in (rnd(B, T, C), rnd(B, T, C), rnd(B, 3, C), rnd(B, 3, C)))
    w, bias = rnd(C, 4).to(dt), rnd(C).to(dt)
    desc = block._conv_desc(x, w, bias, "silu", S, None, None)
    row = lambda t: block._conv_rows(t, x, "t")  # noqa: E731
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    shapes = dict(dx=x, dw=torch.empty((C, 4), device="cuda"), db=torch.empty(C, device="cuda"), ds=S)

    def back(left, dS):
        got = {k: torch.full_like(t, NAN) for k, t in shapes.items() if k not in left}
        ws = _ws(block.short_conv_workspace_bytes(B, T, C, 4, dt))
        block._call("dla_short_conv_backward", x.device, desc, row(x), w.data_ptr(), bias.data_ptr(), S.data_ptr(), row(dy), ptr(dS),
                    row(got["dx"]), got["dw"].data_ptr(), ptr(got.get("db")), ptr(got.get("ds")), ws.data_ptr(), ws.numel())
        return got

    for g in (dS, None):
        want = back((), g)
        for t in want.values():
            assert torch.isfinite(t).all()
        for left in (("db",), ("ds",), ("db", "ds")):
            got = back(left, g)
            _same(got, want, got)
    zero = back((), torch.zeros_like(dS))
    _same(back((), None), zero, zero)
    out, last = block.short_conv(x, w, bias, state=S, want_state=True)
    assert torch.equal(block.short_conv(x, w, bias, state=S)[0], out)
    S0 = torch.zeros_like(S)
    a, b = block.short_conv(x, w, bias, state=S0, want_state=True), block.short_conv(x, w, bias, want_state=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V,top", [(3, 500, 4), (600, 900, 3), (2, 70000, 20)])
def test_log_probabilities(N, V, top, dtype):
    block, rnd, dt = _block(), _rnd(V), DT[dtype]
    l = (3 * rnd(N, V)).to(dt)
    tok = torch.randint(0, V, (N,), device="cuda")
    tok[0] = -1
    row = block._logit_rows(l, "l")
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731

    def forward(names, top):
        f = lambda *s: torch.full(s, NAN, device="cuda")  # noqa: E731
        got = {k: f(N) for k in names}
        if top:
            got["ids"], got["tops"] = torch.full((N, top), -7, device="cuda"), f(N, top)
        desc = block._LOGPROBS.pack(N, V, top, block._code(dt))
        ws = _ws(block._logprobs_bytes(N, V, top, dt))
        block._call("dla_token_logprobs", l.device, desc, row, tok.data_ptr(), *(ptr(got.get(k)) for k in ("lp", "lse", "ent", "ids", "tops")),
                    ws.data_ptr(), ws.numel())
        return got

    for t in (0, top):
        want = forward(("lp", "lse", "ent"), t)
        for names in (("lp",), ("lse",), ("ent",), ("lp", "ent"), ()):
            got = forward(names, t)
            # (without entropies the sums are another kernel's, in the same order)
            _same(got, want, got)
    whole = forward(("lp", "lse", "ent"), 0)
    lp, lse, ent = (whole[k] for k in ("lp", "lse", "ent"))
    a, b, c = rnd(N), rnd(N), rnd(N)
    zero = torch.zeros(N, device="cuda")
    back = lambda dlp, dent, dlse: block.token_logprobs_backward(l, tok, lp, lse, dlp, entropy=ent, dentropy=dent, dlse=dlse)  # noqa: E731
    for g in ((a, None, None), (None, b, None), (None, None, c), (a, b, None), (a, None, c), (None, b, c), (None, None, None)):
        assert torch.equal(back(*g), back(*(zero if t is None else t for t in g)))
