"""dla_train.h without a GPU: it compiles as C, its size queries answer, and arguments are
refused by status before anything touches a device."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2606_10650_amd import dla, train

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000
BF16, F32 = torch.bfloat16, torch.float32


def test_header_compiles_as_c(tmp_path):
    c = tmp_path / "t.c"
    c.write_text('#include "dla_train.h"\nint main(void){dla_recurrence_desc d={1,1,1,1,64,64,DLA_BF16,1.f,0};'
                 'dla_adamw_tensor t={0};dla_norm_desc n={0};(void)d;(void)t;(void)n;return DLA_STATE_FP8-2;}\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-fsyntax-only",
                    str(c)], check=True)


def test_packed_arguments_match_the_header(tmp_path):
    """The sizes of the bytes that the binding packs, against the C structures."""
    c = tmp_path / "s.c"
    c.write_text('#include <stdio.h>\n#include "dla_train.h"\nint main(void){printf("%zu %zu %zu %zu %zu %zu",'
                 'sizeof(dla_rows),sizeof(dla_recurrence_desc),sizeof(dla_norm_desc),sizeof(dla_norm_rows),'
                 'sizeof(dla_adamw_tensor),sizeof(dla_adamw_params));return 0;}\n')
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(c), "-o", str(exe)], check=True)
    sizes = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    have = [train._ROWS.size, train._RECURRENCE.size, train._NORM.size, train._NORM_ROWS.size,
            ctypes.sizeof(train.AdamWTensor), ctypes.sizeof(train.AdamWParams)]
    # (a packed structure may lack the padding at its end)
    assert all(h == s or s - 8 < h < s for h, s in zip(have, sizes)), (have, sizes)


@pytest.mark.parametrize("backward", [False, True])
def test_workspace_sizes(backward):
    size = lambda B, H, Hk, T, dt=BF16: train.recurrence_workspace_bytes(B, H, Hk, T, 64, 128, dt, backward=backward)  # noqa: E731
    assert size(0, 4, 4, 100) == 0 and size(2, 4, 4, 0) == 0
    assert (size(1, 1, 1, 1) > 0) == backward           # a few tokens forward need none
    for T in (1, 31, 33, 1000, 100000):
        for B, H in ((1, 1), (3, 7), (64, 64)):
            assert size(B, H, H, T) <= size(B, H, H, 2 * T)
            assert size(B, H, H, T) % 256 == 0
    assert size(1, 4, 1, 100) > size(1, 4, 4, 100) or not backward
    assert train.rms_norm_workspace_bytes(0, 64) == 0 < train.rms_norm_workspace_bytes(1, 64)


def test_descriptor_refusals():
    n = ctypes.c_size_t(0)
    ask = lambda *a: train.lib().dla_recurrence_workspace_size(train._desc(*a), 0, ctypes.byref(n))  # noqa: E731
    for bad in ((-1, 1, 1, 8, 64, 64, BF16), (1, 0, 1, 8, 64, 64, BF16), (1, 4, 3, 8, 64, 64, BF16),
                (1, 2, 4, 8, 64, 64, BF16), (1, 1, 1, -1, 64, 64, BF16)):
        assert ask(*bad) == dla.DLA_ERR_INVALID_ARG
        assert train.lib().dla_get_last_error() == dla.DLA_ERR_INVALID_ARG
    for bad in ((1, 1, 1, 8, 32, 64, BF16), (1, 1, 1, 8, 64, 256, BF16), (1 << 14, 8, 8, 8, 64, 64, F32),
                (1, 1, 1, (1 << 30) + 1, 64, 64, F32)):
        assert ask(*bad) == dla.DLA_ERR_UNSUPPORTED
    assert ask(1, 1, 1, 8, 64, 64, F32) == dla.DLA_OK
    assert train.lib().dla_recurrence_workspace_size(None, 0, ctypes.byref(n)) == dla.DLA_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        train._desc(1, 1, 1, 8, 64, 64, torch.float16)


def test_call_refusals():
    """Null pointers, bases and strides off their alignment, missing workspaces."""
    L = train.lib()
    desc = train._desc(1, 2, 2, 40, 64, 64, BF16)
    rows = lambda p=FAKE, b=0, h=64, t=128: train._ROWS.pack(p, b, h, t)  # noqa: E731
    ok, gate = rows(), rows(h=1, t=2)

    def fwd(q=ok, k=ok, v=ok, g=gate, S=None, out=ok, last=None, ws=FAKE, size=1 << 30, d=desc):
        return L.dla_recurrence_forward(d, q, k, v, g, S, out, last, ws, size, None)

    for kw in (dict(q=None), dict(k=rows(0)), dict(v=rows(FAKE + 8)), dict(out=rows(t=130)), dict(out=rows(t=0)),
               dict(out=rows(h=32)), dict(g=rows(FAKE + 2, h=1, t=2)), dict(S=FAKE + 4), dict(last=FAKE + 8),
               dict(q=rows(t=-128)), dict(q=rows(t=1 << 26)), dict(d=None)):
        assert fwd(**kw) == dla.DLA_ERR_INVALID_ARG, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 16), dict(size=255)):
        assert fwd(**kw) == dla.DLA_ERR_WORKSPACE, kw
    back = [desc, ok, ok, ok, gate, None, ok, None, ok, ok, ok, gate, None, FAKE, 1 << 30, None]
    for i, bad in ((6, None), (8, None), (9, rows(t=64)), (10, rows(FAKE + 1)), (11, rows(h=0, t=2)), (12, FAKE + 4)):
        a = list(back)
        a[i] = bad
        assert L.dla_recurrence_backward(*a) == dla.DLA_ERR_INVALID_ARG, i
    assert L.dla_recurrence_backward(*back[:13], None, 0, None) == dla.DLA_ERR_WORKSPACE


def test_norm_refusals():
    L = train.lib()
    nd = lambda rows=4, D=64, dt=1, w=1, eps=1e-6: train._NORM.pack(rows, D, dt, w, eps)  # noqa: E731
    r = lambda p=FAKE, s=64: train._NORM_ROWS.pack(p, s)  # noqa: E731
    assert L.dla_rms_norm(nd(0), None, None, FAKE, None, None, None, None) == dla.DLA_OK
    for d in (nd(-1), nd(D=0), nd(dt=7), nd(dt=0, w=1), nd(eps=-1.0), nd(eps=float("nan"))):
        assert L.dla_rms_norm(d, r(), None, FAKE, None, r(), None, None) == dla.DLA_ERR_INVALID_ARG
    assert L.dla_rms_norm(nd(D=16385), r(s=20000), None, FAKE, None, r(s=20000), None, None) == dla.DLA_ERR_UNSUPPORTED
    for x, w, y in ((None, FAKE, r()), (r(), None, r()), (r(), FAKE, None), (r(s=63), FAKE, r()), (r(FAKE + 1), FAKE, r())):
        assert L.dla_rms_norm(nd(), x, None, w, None, y, None, None) == dla.DLA_ERR_INVALID_ARG
    assert L.dla_rms_norm_fp8(nd(), r(), None, FAKE, None, r(), None, None) == dla.DLA_ERR_INVALID_ARG   # no scales
    assert L.dla_rms_norm_backward(nd(), r(), r(), FAKE, None, None, r(), None, None, 0, None) == dla.DLA_ERR_INVALID_ARG
    assert L.dla_rms_norm_backward(nd(), r(), r(), FAKE, FAKE, None, r(), FAKE, None, 0, None) == dla.DLA_ERR_WORKSPACE


def test_adamw_refusals():
    L = train.lib()
    T, P = train.AdamWTensor, train.AdamWParams

    def step(t=None, n=1, **kw):
        p = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, param_dtype=0, grad_dtype=0, state_format=0, seed=0,
                 grad_scale=None)
        p.update(kw)
        arr = (T * 1)(t or T(FAKE, None, FAKE, FAKE, FAKE, None, None, 0, 0.0))
        return L.dla_adamw_step(arr, n, ctypes.byref(P(**p)), None)

    assert step() == dla.DLA_OK                                 # a tensor without elements
    assert step(n=0) == dla.DLA_OK
    for kw in (dict(n=-1), dict(step=0), dict(beta1=1.0), dict(beta2=float("nan")), dict(eps=-1.0),
               dict(lr=float("inf")), dict(param_dtype=3), dict(grad_dtype=-1), dict(state_format=1),
               dict(grad_scale=FAKE + 2)):
        assert step(**kw) == dla.DLA_ERR_INVALID_ARG, kw
    full = lambda **kw: T(**{**dict(param=FAKE, master=None, grad=FAKE, m=FAKE, v=FAKE, m_scale=None, v_scale=None, n=5,  # noqa: E731
                                    weight_decay=0.0), **kw})
    for kw in (dict(param=None), dict(grad=None), dict(m=None), dict(v=FAKE + 1), dict(master=FAKE + 2),
               dict(param=FAKE + 2), dict(n=-1), dict(n=(1 << 40) + 1), dict(weight_decay=float("nan"))):
        assert step(full(**kw)) == dla.DLA_ERR_INVALID_ARG, kw
    assert step(full(), state_format=train.DLA_STATE_FP8) == dla.DLA_ERR_INVALID_ARG    # no scales
