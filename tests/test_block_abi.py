"""dla_block.h without a GPU: it compiles as C, its size queries answer, and arguments are refused by status,
or by the binding, before anything touches a device."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2606_10650_amd import block, dla

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000
BF16, F32 = torch.bfloat16, torch.float32
OK, BAD, NO, SPACE = dla.DLA_OK, dla.DLA_ERR_INVALID_ARG, dla.DLA_ERR_UNSUPPORTED, dla.DLA_ERR_WORKSPACE
NAN, INF = float("nan"), float("inf")


def test_packed_arguments_match_the_header(tmp_path):
    c = tmp_path / "s.c"
    names = ("dla_conv_desc", "dla_conv_rows", "dla_gated_norm_desc", "dla_group_rows", "dla_logprobs_desc", "dla_ff_desc",
             "dla_norm_rows")
    c.write_text('#include <stdio.h>\n#include "dla_block.h"\nint main(void){' +
                 "".join(f'printf("%zu ",sizeof({n}));' for n in names) + 'return 0;}\n')
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(c), "-o", str(exe)],
                   check=True)
    sizes = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    have = [s.size for s in (block._CONV, block._CONV_ROWS, block._NORM, block._GROUP_ROWS, block._LOGPROBS, block._FF,
                             block._ROWS)]
    # (a packed structure may lack the padding at its end)
    assert all(h == s or s - 8 < h < s for h, s in zip(have, sizes)), (have, sizes)


def conv(B=2, T=5, C=8, W=4, dt=1, wt=1, silu=1, lengths=0, starts=0):
    return block._CONV.pack(B, T, C, W, dt, wt, silu, lengths, starts)


def test_conv_refusals():
    L, n = block.lib(), ctypes.c_size_t(0)
    ask = lambda d: L.dla_short_conv_workspace_size(d, ctypes.byref(n))  # noqa: E731
    for d in (conv(B=-1), conv(T=-1), conv(C=-1), conv(dt=2), conv(dt=0, wt=1), conv(silu=2), conv(lengths=FAKE + 2), None):
        assert ask(d) == BAD
    for d in (conv(W=1), conv(W=5), conv(T=(1 << 30) + 1), conv(C=(1 << 30) + 1)):
        assert ask(d) == NO
    assert ask(conv()) == OK and n.value > 0 and L.dla_short_conv_workspace_size(conv(), None) == BAD
    for d in (conv(B=0), conv(T=0), conv(C=0)):
        assert ask(d) == OK
    r = lambda p=FAKE, b=40, t=8: block._CONV_ROWS.pack(p, b, t)  # noqa: E731

    def fwd(d=conv(), x=r(), w=FAKE, bias=None, S=None, y=r(), last=None):
        return L.dla_short_conv(d, x, w, bias, S, y, last, None)

    for kw in (dict(x=None), dict(x=r(0)), dict(x=r(FAKE + 1)), dict(w=None), dict(w=FAKE + 1), dict(bias=FAKE + 1),
               dict(S=FAKE + 1), dict(last=FAKE + 1), dict(y=None), dict(y=r(t=7)), dict(y=r(b=39)), dict(y=r(b=0)),
               dict(x=r(t=-8)), dict(d=None)):
        assert fwd(**kw) == BAD, kw
    assert fwd(d=conv(B=0), x=None, y=None) == OK and fwd(d=conv(T=0), x=None, y=None) == OK
    # a launch has fewer than 2^32 threads
    assert fwd(d=conv(B=(1 << 31) - 1, T=1, C=64), x=r(b=0), y=r(b=64)) == NO

    def back(d=conv(), x=r(), w=FAKE, dy=r(), dS=None, dx=r(), dw=FAKE, db=None, ds=None, ws=FAKE, size=1 << 20):
        return L.dla_short_conv_backward(d, x, w, None, None, dy, dS, dx, dw, db, ds, ws, size, None)

    for kw in (dict(x=None), dict(dy=None), dict(dx=r(t=0)), dict(dw=None), dict(dw=FAKE + 2), dict(db=FAKE + 2),
               dict(dS=FAKE, ds=FAKE), dict(w=None)):
        assert back(**kw) == BAD, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 16), dict(size=10)):
        assert back(**kw) == SPACE, kw


def gnorm(rows=4, G=2, D=8, dt=1, wt=1, per_group=0, eps=1e-6, scale=1.0):
    return block._NORM.pack(rows, G, D, dt, wt, per_group, eps, scale)


def test_gated_norm_refusals():
    L, n = block.lib(), ctypes.c_size_t(0)
    ask = lambda d: L.dla_gated_norm_workspace_size(d, ctypes.byref(n))  # noqa: E731
    for d in (gnorm(rows=-1), gnorm(G=0), gnorm(D=0), gnorm(dt=3), gnorm(dt=0, wt=1), gnorm(per_group=2), gnorm(eps=-1.0),
              gnorm(eps=NAN), gnorm(scale=INF), gnorm(scale=NAN), None):
        assert ask(d) == BAD
    for d in (gnorm(D=16385), gnorm(G=65536), gnorm(G=65535, D=2048), gnorm(rows=(1 << 31) - 3)):
        assert ask(d) == NO
    for kw in (dict(rows=0), dict(G=65535, D=1024), dict(rows=(1 << 31) - 4), dict(per_group=1)):
        assert ask(gnorm(**kw)) == OK
        assert (n.value > 0) == (kw.get("rows") != 0) and n.value < 1 << 30
    r = lambda p=FAKE, s=16, g=8: block._GROUP_ROWS.pack(p, s, g)  # noqa: E731

    def fwd(d=gnorm(), x=r(), gate=None, res=None, w=FAKE, w2=None, h=r(), y=None, rstd=None, y_rstd=None):
        return L.dla_gated_norm(d, x, gate, res, w, w2, h, y, rstd, y_rstd, None)

    one = gnorm(G=1)
    for kw in (dict(x=None), dict(x=r(FAKE + 1)), dict(gate=r(0)), dict(res=r(s=-1)), dict(w=None), dict(h=None),
               dict(h=r(s=15)), dict(h=r(g=7)), dict(h=r(g=0)), dict(h=r(s=0)), dict(w2=FAKE), dict(d=one, w2=FAKE), dict(rstd=FAKE + 2),
               dict(d=one, w2=FAKE, y=r(s=7)), dict(d=one, w2=FAKE, y=r(), y_rstd=FAKE + 1)):
        assert fwd(**kw) == BAD, kw
    assert fwd(d=gnorm(rows=0), x=None, h=None) == OK

    def back(d=one, x=r(), gate=None, res=None, w=FAKE, w2=None, rstd=FAKE, y_rstd=FAKE, dh=r(), dy=None, dx=r(), dgate=None,
             dres=None, dw=FAKE, dw2=None, ws=FAKE, size=1 << 20):
        return L.dla_gated_norm_backward(d, x, gate, res, w, w2, rstd, y_rstd, dh, dy, dx, dgate, dres, dw, dw2, ws, size, None)

    for kw in (dict(x=None), dict(w=None), dict(rstd=None), dict(dx=None), dict(dx=r(s=0)), dict(dgate=r()), dict(dy=r()), dict(dw2=FAKE),
               dict(w2=FAKE, dy=r(), y_rstd=None), dict(dh=r(0)), dict(dres=r(FAKE + 1)), dict(d=gnorm(), w2=FAKE)):
        assert back(**kw) == BAD, kw
    for kw in (dict(ws=None), dict(size=16), dict(ws=FAKE + 8)):
        assert back(**kw) == SPACE, kw


def lps(rows=3, V=10, top=0, dt=1):
    return block._LOGPROBS.pack(rows, V, top, dt)


def test_logprobs_refusals():
    L, n = block.lib(), ctypes.c_size_t(0)
    ask = lambda d: L.dla_token_logprobs_workspace_size(d, ctypes.byref(n))  # noqa: E731
    for d in (lps(rows=-1), lps(V=0), lps(top=-1), lps(top=11), lps(dt=5), None):
        assert ask(d) == BAD
    for d in (lps(rows=1 << 31), lps(V=(1 << 30) + 1), lps(V=100, top=65)):
        assert ask(d) == NO
    assert ask(lps(rows=0)) == OK and ask(lps(V=100, top=64)) == OK
    r = lambda p=FAKE, s=10: block._ROWS.pack(p, s)  # noqa: E731

    def fwd(d=lps(), l=r(), tok=FAKE, lp=FAKE, lse=None, ent=None, ids=None, tops=None):
        return L.dla_token_logprobs(d, l, tok, lp, lse, ent, ids, tops, None, 0, None)

    for kw in (dict(l=None), dict(l=r(FAKE + 1)), dict(l=r(s=-1)), dict(tok=None), dict(tok=FAKE + 4), dict(lp=FAKE + 2), dict(lse=FAKE + 1),
               dict(ent=FAKE + 1), dict(d=lps(top=2)), dict(d=lps(top=2), ids=FAKE), dict(d=lps(top=2), ids=FAKE + 4, tops=FAKE), dict(d=None)):
        assert fwd(**kw) == BAD, kw
    assert fwd(d=lps(rows=0), l=None) == OK

    def back(d=lps(), l=r(), tok=FAKE, lp=FAKE, lse=FAKE, ent=FAKE, dlp=FAKE, dent=FAKE, dlse=None, dl=r()):
        return L.dla_token_logprobs_backward(d, l, tok, lp, lse, ent, dlp, dent, dlse, dl, None)

    for kw in (dict(l=None), dict(dl=None), dict(dl=r(s=9)), dict(lse=None), dict(tok=None), dict(lp=None), dict(ent=None), dict(dlse=FAKE + 1)):
        assert back(**kw) == BAD, kw
    assert back(d=lps(rows=0), l=None, dl=None) == OK


def ff(rows=100, D=16, F=24, dt=1):
    return block._FF.pack(rows, D, F, dt)


def test_gated_ff_refusals():
    L, n = block.lib(), ctypes.c_size_t(0)

    def ask(d, backward=0, aligned=1):
        return L.dla_gated_ff_workspace_size(d, backward, aligned, ctypes.byref(n))

    for d in (ff(rows=-1), ff(D=0), ff(F=0), ff(dt=9), None):
        assert ask(d) == BAD
    for d in (ff(rows=(1 << 30) + 1), ff(D=65537), ff(F=65537)):
        assert ask(d) == NO
    for rows in (0, 1, 64, 65, 5000, 100000):
        for D, F in ((16, 24), (15, 24), (16, 23), (2048, 5504)):
            for dt in (0, 1):
                assert ask(ff(rows, D, F, dt)) == OK
                if rows <= 64:
                    assert n.value == 0
                elif dt == 0 or D % 8:
                    assert n.value >= (rows + 2 * F) * D * 2
                assert ask(ff(rows, D, F, dt), 0, 0) == OK and (n.value > 0) == (rows > 64)
                assert ask(ff(rows, D, F, dt), 1) == OK and n.value >= rows * F * 4
    r = lambda p=FAKE, s=24: block._ROWS.pack(p, s)  # noqa: E731

    def fwd(d=ff(), x=r(), wg=r(), wu=r(), y=r(), g=None, u=None, ws=FAKE, size=1 << 30):
        return L.dla_gated_ff(d, x, wg, wu, y, g, u, ws, size, None)

    for kw in (dict(x=None), dict(x=r(0)), dict(wg=r(FAKE + 1)), dict(wu=None), dict(y=None), dict(y=r(s=23)), dict(g=r()), dict(u=r()),
               dict(x=r(s=-1)), dict(d=None)):
        assert fwd(**kw) == BAD, kw
    assert fwd(d=ff(rows=0), x=None, y=None) == OK
    odd = r(FAKE + 2)
    for kw in (dict(x=odd, size=100), dict(wg=odd, ws=None), dict(wu=odd, ws=FAKE + 16), dict(d=ff(dt=0), size=100),
               dict(wu=r(s=32), size=100)):
        assert fwd(**kw) == SPACE, kw

    def back(d=ff(), x=r(), wg=r(), wu=r(), g=r(), u=r(), dy=r(), dx=r(), dwg=r(), dwu=r(), ws=FAKE, size=1 << 30):
        return L.dla_gated_ff_backward(d, x, wg, wu, g, u, dy, dx, dwg, dwu, ws, size, None)

    for kw in (dict(x=None), dict(wg=None), dict(g=None), dict(u=r(FAKE + 1)), dict(dy=None), dict(dx=r(s=15)), dict(dwg=r(s=8)),
               dict(dwu=r(0)), dict(d=None)):
        assert back(**kw) == BAD, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 128), dict(size=1000)):
        assert back(**kw) == SPACE, kw


def test_binding_refusals():
    """Shapes, types, layouts and devices that do not fit, before the library is called."""
    z = torch.zeros
    x, w = z(2, 5, 8), z(8, 4)
    meta = torch.device("meta")
    for a, kw in (((z(5, 8), w), {}), ((x, z(8)), {}), ((x, z(7, 4)), {}), ((x, w.to(BF16)), {}), ((x, w, z(7)), {}),
                  ((x, w, z(8, dtype=BF16)), {}), ((x, w), dict(activation="gelu")), ((x, w), dict(state=z(2, 4, 8))),
                  ((x, w), dict(state=z(2, 3, 8, dtype=BF16))), ((x, w), dict(lengths=z(2))), ((x, w), dict(starts=z(2, 5))),
                  ((x, w), dict(starts=z(5, 2, dtype=torch.bool).t())), ((x, w), dict(out=z(2, 5, 9))),
                  ((x.transpose(1, 2).contiguous().transpose(1, 2), w), {}), ((x, w), dict(state_out=z(2, 3, 8, device=meta)))):
        with pytest.raises(ValueError):
            block.short_conv(*a, **kw)
    with pytest.raises(ValueError):
        block.short_conv_backward(x, w, z(2, 5, 8, dtype=BF16))
    x, w = z(6, 2, 8), z(8)
    for a, kw in (((z(8), w), {}), ((x, z(7)), {}), ((x, z(3, 8)), {}), ((x, w, z(6, 2, 7)), {}), ((x, w, None, z(6, 2, 8, dtype=BF16)), {}),
                  ((x, w), dict(next_weight=w)), ((x[:, 0], w), dict(next_weight=z(8, dtype=BF16))),
                  ((x.transpose(1, 2).contiguous().transpose(1, 2), w), {})):
        with pytest.raises(ValueError):
            block.gated_norm(*a, **kw)
    rows, r = z(6, 8), z(6, 1)
    for kw in (dict(dy=rows), dict(dy=rows, next_weight=w), dict(dy=rows, next_weight=w, y_rstd=z(5))):
        with pytest.raises(ValueError):
            block.gated_norm_backward(rows, rows, w, r, **kw)
    with pytest.raises(ValueError):
        block.gated_norm_backward(rows, rows, w, z(6))
    l, tok = z(3, 10), z(3, dtype=torch.int64)
    for a, kw in (((z(10), tok), {}), ((l, z(4, dtype=torch.int64)), {}), ((l, z(3, dtype=torch.int32)), {}), ((l.t(), z(10, dtype=torch.int64)), {}),
                  ((l.to(torch.float16), tok), {})):
        with pytest.raises(ValueError):
            block.token_logprobs(*a, **kw)
    with pytest.raises(dla.DLAError):
        block.token_logprobs(l, tok, top=11)
    with pytest.raises(ValueError):
        block.token_logprobs_backward(l, tok, z(3), z(3), z(4))
    x, w = z(5, 16), z(24, 16)
    for a, kw in (((x, z(24, 15), w), {}), ((x, w, z(23, 16)), {}), ((x, w.to(BF16), w), {}), ((x, w.t().contiguous().t(), w), {}),
                  ((x, w, w), dict(out=z(5, 23))), ((z(16), w, w), {})):
        with pytest.raises(ValueError):
            block.gated_ff(*a, **kw)
    with pytest.raises(ValueError):
        block.gated_ff_backward(x, w, w, z(2, 5, 23), z(5, 24))
    with pytest.raises(ValueError):
        block.gated_ff_backward(x, w, w, z(2, 5, 24), z(5, 23))
    with pytest.raises(ValueError):
        block.gated_ff_backward(x, w, w, z(2, 5, 24, dtype=BF16), z(5, 24))


def test_outputs_apart_from_inputs():
    """An output in an input's place is refused: other runs and tiles still read it."""
    x, w = torch.zeros(1, 8, 16), torch.zeros(16, 4)
    with pytest.raises(ValueError, match="array of an input"):
        block.short_conv(x, w, out=x)
    a, g = torch.zeros(4, 16), torch.zeros(16, 16)
    for out in (a, g[:4]):
        with pytest.raises(ValueError, match="array of an input"):
            block.gated_ff(a, g, torch.zeros(16, 16), out=out)
