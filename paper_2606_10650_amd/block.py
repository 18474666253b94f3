"""Python binding of libdla's operators around the recurrence (include/dla_block.h): the short
causal convolution in front of it, the norm with gate, residual sum and next norm behind it,
the gated feed-forward block, and the log probabilities of tokens.  Argument marshalling only:
the work is the library's, torch provides device memory and the current stream.

Below the calls, the same as differentiable functions (`ShortConv`, `GatedNorm`, `GatedFF`,
`TokenLogprobs`) for a model written in torch.
"""
from __future__ import annotations

import ctypes
import functools
import math
import struct
from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import train
from .dla import EXPORTED, _check, _dtype_code
from .train import _like, _ptr, _run, _space

# descriptions of arguments, packed as bytes (see train.py)
_CONV = struct.Struct("7iPP")            # dla_conv_desc
_CONV_ROWS = struct.Struct("Pqq")        # dla_conv_rows
_NORM = struct.Struct("q5iff")           # dla_gated_norm_desc
_GROUP_ROWS = struct.Struct("Pqq")       # dla_group_rows
_LOGPROBS = struct.Struct("q3i")         # dla_logprobs_desc
_FF = struct.Struct("q3i")               # dla_ff_desc
_ROWS = struct.Struct("Pq")              # dla_norm_rows

_code = functools.lru_cache(maxsize=None)(_dtype_code)   # a dictionary's look-up


@functools.lru_cache(maxsize=None)
def lib():
    """libdla.so with the entry points of dla_block.h declared."""
    L = train.lib()
    P, S, I = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    size = ctypes.POINTER(S)
    L.dla_short_conv.argtypes = [P] * 8
    L.dla_short_conv_workspace_size.argtypes = [P, size]
    L.dla_short_conv_backward.argtypes = [P] * 12 + [S, P]
    L.dla_gated_norm.argtypes = [P] * 11
    L.dla_gated_norm_workspace_size.argtypes = [P, size]
    L.dla_gated_norm_backward.argtypes = [P] * 16 + [S, P]
    L.dla_token_logprobs_workspace_size.argtypes = [P, size]
    L.dla_token_logprobs.argtypes = [P] * 9 + [S, P]
    L.dla_token_logprobs_backward.argtypes = [P] * 11
    L.dla_gated_ff_workspace_size.argtypes = [P, I, I, size]
    L.dla_gated_ff.argtypes = [P] * 8 + [S, P]
    L.dla_gated_ff_backward.argtypes = [P] * 11 + [S, P]
    for name in EXPORTED:
        if name.startswith(("dla_short_conv", "dla_gated", "dla_token_logprobs")):
            getattr(L, name).restype = ctypes.c_int
    return L


def _call(call, device, *args):
    lib()
    _run(call, device, *args)


def _bytes(call, *args):
    n = ctypes.c_size_t(0)
    _check(getattr(lib(), call)(*args, ctypes.byref(n)), call)
    return int(n.value)


def _work(workspace, need, device):
    """A workspace and its size, where one is needed."""
    return _space(workspace, need, device) if need else (None, 0)


def _new(t):
    """A contiguous tensor like t."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _last(t, name):
    if t.stride(-1) != 1 and t.shape[-1] > 1 and t.numel():
        raise ValueError(f"{name}: the last axis must be contiguous")


def _place(t):
    """Where a tensor's elements lie: the first byte, and counts and distances in bytes of what repeats, the furthest
    apart first; the last is a run of bytes."""
    e, run, more = t.element_size(), 1, []
    for distance, n in sorted(zip(t.stride(), t.shape)):
        if distance == run and not more:
            run *= n
        elif n > 1 and distance:
            more.append((n, distance * e))
    return t.data_ptr(), (*reversed(more), (run * e, 1))


def _meet(off, a, b):
    """Whether a byte is both what lies as `a` and what lies as `b` and begins `off` bytes behind it; also where that is not
    told by their distances."""
    ends = [sum((n - 1) * s for n, s in t) + 1 for t in (a, b)]
    if off >= ends[0] or off + ends[1] <= 0:
        return False
    (n, s), (m, t) = a[0], b[0]
    if s == t == 1:
        return True
    if s == t:
        # rows of one distance: those near each other
        each = [end - (k - 1) * s for end, k in zip(ends, (n, m))]
        low, high = max(1 - n, (-each[1] - off) // s + 1), min(m - 1, (each[0] - off - 1) // s)
        if high - low < 8:
            return any(_meet(off + k * s, a[1:], b[1:]) for k in range(low, high + 1))
    # runs at multiples of a common step
    step = functools.reduce(math.gcd, [s for _, s in (*a[:-1], *b[:-1])])
    return off % step < a[-1][0] or off % step + b[-1][0] > step


def _apart(name, out, *inputs):
    """An output whose elements are no input's: those are still read when the first results are written.  Columns or
    tokens of one wider array are apart."""
    if not out.numel():
        return
    at, own = _place(out)
    for t in inputs:
        if t is not None and t.numel():
            t_at, t_own = _place(t)
            if _meet(t_at - at, own, t_own):
                raise ValueError(f"{name}: lies over the array of an input")


def _weight(t, shape, like, name, code=None):
    """The type code of a contiguous weight of the given shape: the inputs' type or float32."""
    dtype = t.dtype
    if t.shape != shape or not t.is_contiguous() or t.device != like.device or \
            (dtype != like.dtype and dtype != torch.float32):
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, not contiguous {like.dtype} or float32 "
                         f"{tuple(shape)} on {like.device}")
    own = _code(dtype)
    if code is not None and own != code:
        raise ValueError(f"{name}: {dtype}: weights of one type are wanted")
    return own


# ---------------------------------------------------------------------------
# short causal convolution
# ---------------------------------------------------------------------------
_ACTIVATIONS = {None: 0, "silu": 1}


def _conv_desc(x, weight, bias, activation, state, lengths, starts):
    if x.dim() != 3 or weight.dim() != 2:
        raise ValueError(f"shapes {tuple(x.shape)}, {tuple(weight.shape)}: x [B, T, C] and a weight [C, W] are wanted")
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation {activation!r}: silu or None")
    B, T, C = x.shape
    W, dev = weight.shape[1], x.device
    code = _weight(weight, (C, W), x, "weight")
    if bias is not None:
        _weight(bias, (C,), x, "bias", code)
    _like(state, (B, W - 1, C), x.dtype, dev, "state", True)
    _like(lengths, (B,), torch.int32, dev, "lengths", True)
    if starts is not None and starts.dtype == torch.bool:
        starts = starts.view(torch.uint8)
    _like(starts, (B, T), torch.uint8, dev, "starts", True)
    return _CONV.pack(B, T, C, W, _code(x.dtype), code, _ACTIVATIONS[activation],
                      0 if lengths is None else lengths.data_ptr(), 0 if starts is None else starts.data_ptr())


def _conv_rows(t, like, name):
    _like(t, like.shape, like.dtype, like.device, name)
    _last(t, name)
    return _CONV_ROWS.pack(t.data_ptr(), t.stride(0), t.stride(1))


def short_conv(x, weight, bias=None, *, activation: Optional[str] = "silu", state=None, state_out=None,
               want_state: bool = False, lengths=None, starts=None, out=None):
    """z_t = bias + sum_j weight[:, j] x_{t - (W - 1) + j} per channel, and its SiLU (dla_short_conv).
    x: [B, T, C], last axis contiguous; weight [C, W], W 2 to 4; state [B, W - 1, C], the inputs before
    the call, or None; lengths int32 [B]; starts [B, T], bool or uint8, where documents start.  state_out
    may be state; otherwise state_out and out are apart from the inputs and each other.  Returns (out, state_out);
    out is contiguous unless given."""
    desc = _conv_desc(x, weight, bias, activation, state, lengths, starts)
    B, T, C = x.shape
    _last(x, "x")
    at, (b, t, _) = x.data_ptr(), x.stride()
    given = out
    if out is None:
        out = _new(x)
        rows = _CONV_ROWS.pack(out.data_ptr(), T * C, C)
    else:
        rows = _conv_rows(out, x, "out")
        _apart("out", out, x, weight, bias, state, lengths, starts)
    if state_out is not None:
        if state_out is not state:
            _like(state_out, (B, weight.shape[1] - 1, C), x.dtype, x.device, "state_out", True)
            same = state is not None and state.data_ptr() == state_out.data_ptr()
            _apart("state_out", state_out, weight, bias, lengths, starts, given, None if same else state)
        # (mostly told by their ends)
        e, s = x.element_size(), state_out.data_ptr()
        if at < s + state_out.numel() * e and s < at + ((B - 1) * b + (T - 1) * t + C) * e:
            _apart("state_out", state_out, x)
    elif want_state:
        state_out = x.new_empty((B, weight.shape[1] - 1, C))
    _call("dla_short_conv", x.device, desc, _CONV_ROWS.pack(at, b, t), weight.data_ptr(), _ptr(bias), _ptr(state), rows,
          _ptr(state_out))
    return out, state_out


@functools.lru_cache(maxsize=4096)
def short_conv_workspace_bytes(B: int, T: int, C: int, W: int, dtype=torch.bfloat16) -> int:
    """Workspace of short_conv_backward."""
    code = _code(dtype)
    return _bytes("dla_short_conv_workspace_size", _CONV.pack(B, T, C, W, code, code, 0, 0, 0))


def short_conv_backward(x, weight, dout, bias=None, *, activation: Optional[str] = "silu", state=None, dstate=None,
                        lengths=None, starts=None, want_dstate: Optional[bool] = None, workspace=None):
    """Gradients of `short_conv` (dla_short_conv_backward) from those of its outputs, dout and dstate
    (None: zero).  Returns dx, dweight (float32), dbias (float32; None without a bias) and the gradient of
    `state` (None without one, unless want_dstate)."""
    desc = _conv_desc(x, weight, bias, activation, state, lengths, starts)
    (B, T, C), W, dev, f32 = x.shape, weight.shape[1], x.device, torch.float32
    _like(dstate, (B, W - 1, C), x.dtype, dev, "dstate", True)
    dx, dw = _new(x), x.new_empty((C, W), dtype=f32)
    db = None if bias is None else x.new_empty((C,), dtype=f32)
    ds = None
    if state is not None if want_dstate is None else want_dstate:
        ds = x.new_empty((B, W - 1, C))
    workspace, size = _work(workspace, short_conv_workspace_bytes(B, T, C, W, x.dtype), dev)
    _call("dla_short_conv_backward", dev, desc, _conv_rows(x, x, "x"), weight.data_ptr(), _ptr(bias), _ptr(state),
          _conv_rows(dout, x, "dout"), _ptr(dstate), _CONV_ROWS.pack(dx.data_ptr(), T * C, C), dw.data_ptr(), _ptr(db), _ptr(ds),
          _ptr(workspace), size)
    return dx, dw, db, ds


# ---------------------------------------------------------------------------
# norm with gate, residual sum and next norm
# ---------------------------------------------------------------------------
def _group_rows(t, like, name):
    if t is None:
        return None
    _like(t, like.shape, like.dtype, like.device, name)
    _last(t, name)
    st = t.stride()
    return _GROUP_ROWS.pack(t.data_ptr(), st[0], st[1] if len(st) == 3 else 0)


def _gated_desc(x, weight, next_weight, eps, scale):
    if x.dim() not in (2, 3):
        raise ValueError(f"x {tuple(x.shape)}: rows [N, D] or [N, G, D] are wanted")
    N, D = x.shape[0], x.shape[-1]
    G = x.shape[1] if x.dim() == 3 else 1
    per_group = weight.dim() == 2
    code = _weight(weight, (G, D) if per_group else (D,), x, "weight")
    if next_weight is not None:
        _weight(next_weight, (D,), x, "next_weight", code)
        if G != 1:
            raise ValueError("next_weight: a next norm is over rows of one group")
    return _NORM.pack(N, G, D, _code(x.dtype), code, int(per_group), eps, scale)


def gated_norm(x, weight, gate=None, residual=None, *, scale: float = 1.0, next_weight=None, eps: float = 1e-6):
    """n = weight x / rms(x), b = n silu(gate), h = residual + scale b, y = next_weight h / rms(h)
    (dla_gated_norm).  x, gate, residual: [N, D], or [N, G, D] with a norm for each of the G groups (no next
    norm then unless G is 1); weight [D] or [G, D], next_weight [D].  Without gate b = n, without residual it is
    zero, without next_weight y is None.  Returns (h, y, rstd [N, G], y_rstd [N] or None)."""
    desc = _gated_desc(x, weight, next_weight, eps, scale)
    shape = x.shape
    N, D = shape[0], shape[-1]
    G = shape[1] if len(shape) == 3 else 1
    new = lambda t: _GROUP_ROWS.pack(t.data_ptr(), G * D, D)  # noqa: E731
    h, rstd, y, y_rstd = _new(x), x.new_empty((N, G), dtype=torch.float32), None, None
    if next_weight is not None:
        y, y_rstd = _new(x), x.new_empty((N,), dtype=torch.float32)
    _call("dla_gated_norm", x.device, desc, _group_rows(x, x, "x"), _group_rows(gate, x, "gate"),
          _group_rows(residual, x, "residual"), weight.data_ptr(), _ptr(next_weight), new(h),
          None if y is None else new(y), rstd.data_ptr(), _ptr(y_rstd))
    return h, y, rstd, y_rstd


@functools.lru_cache(maxsize=4096)
def gated_norm_workspace_bytes(N: int, G: int, D: int, dtype=torch.bfloat16) -> int:
    """Workspace of gated_norm_backward, whichever weights there are."""
    code = _code(dtype)
    return max(_bytes("dla_gated_norm_workspace_size", _NORM.pack(N, G, D, code, code, per_group, 0.0, 1.0))
               for per_group in (0, 1))


def gated_norm_backward(dh, x, weight, rstd, gate=None, residual=None, *, scale: float = 1.0, next_weight=None, dy=None,
                        y_rstd=None, workspace=None):
    """Gradients of `gated_norm` (dla_gated_norm_backward) from those of its outputs, dh and dy (None: zero), and its
    rstd and y_rstd.  Returns dx, dgate (None without a gate), the residual's gradient (dh itself where there is no
    next norm), dweight and dnext_weight (float32; None without next_weight)."""
    desc = _gated_desc(x, weight, next_weight, 0.0, scale)
    dev, f32, N = x.device, torch.float32, x.shape[0]
    _like(rstd, (N, x.shape[1] if x.dim() == 3 else 1), f32, dev, "rstd", True)
    _like(y_rstd, (N,), f32, dev, "y_rstd", True)
    through = next_weight is not None and dy is not None
    if through and y_rstd is None:
        raise ValueError("dy needs y_rstd")
    if next_weight is None and dy is not None:
        raise ValueError("dy needs next_weight")
    G, D = x.shape[1] if x.dim() == 3 else 1, x.shape[-1]
    dx, dgate, dres = _new(x), None if gate is None else _new(x), _new(x) if through else dh
    dw = x.new_empty(weight.shape, dtype=f32)
    dw2 = None if next_weight is None else x.new_empty(next_weight.shape, dtype=f32)
    new = lambda t: None if t is None else _GROUP_ROWS.pack(t.data_ptr(), G * D, D)  # noqa: E731
    workspace, size = _work(workspace, gated_norm_workspace_bytes(N, G, D, x.dtype), dev)
    _call("dla_gated_norm_backward", dev, desc, _group_rows(x, x, "x"), _group_rows(gate, x, "gate"),
          _group_rows(residual, x, "residual"), weight.data_ptr(), _ptr(next_weight), rstd.data_ptr(), _ptr(y_rstd),
          _group_rows(dh, x, "dh"), _group_rows(dy, x, "dy"), new(dx), new(dgate), new(dres) if through else None,
          dw.data_ptr(), _ptr(dw2), _ptr(workspace), size)
    return dx, dgate, dres, dw, dw2


# ---------------------------------------------------------------------------
# log probabilities
# ---------------------------------------------------------------------------
def _logit_rows(t, name):
    _last(t, name)
    return _ROWS.pack(t.data_ptr(), t.stride(0))


def _logits(logits, tokens, top):
    if logits.dim() != 2:
        raise ValueError(f"logits {tuple(logits.shape)}: rows [N, V] are wanted")
    N, V = logits.shape
    _like(tokens, (N,), torch.int64, logits.device, "tokens", True)
    return _LOGPROBS.pack(N, V, top, _code(logits.dtype))


def token_logprobs(logits, tokens=None, *, top: int = 0, entropy: bool = False, workspace=None):
    """Log probabilities of tokens int64 [N] (negative: none is asked for) under logits [N, V], the rows' entropies, and
    the `top` (at most 64) largest log probabilities with their indices (dla_token_logprobs).  Returns (logprob [N],
    lse [N], entropy [N] or None, ids int64 [N, top] or None, logprobs [N, top] or None), all but ids float32; logprob
    is None without tokens."""
    desc, dev, N = _logits(logits, tokens, top), logits.device, logits.shape[0]
    f = lambda *s: logits.new_empty(s, dtype=torch.float32)  # noqa: E731
    lp, lse, ent = None if tokens is None else f(N), f(N), f(N) if entropy else None
    ids, tops = (logits.new_empty((N, top), dtype=torch.int64), f(N, top)) if top else (None, None)
    workspace, size = _work(workspace, _logprobs_bytes(*logits.shape, top, logits.dtype), dev)
    _call("dla_token_logprobs", dev, desc, _logit_rows(logits, "logits"), _ptr(tokens), _ptr(lp), lse.data_ptr(),
          _ptr(ent), _ptr(ids), _ptr(tops), _ptr(workspace), size)
    return lp, lse, ent, ids, tops


@functools.lru_cache(maxsize=4096)
def _logprobs_bytes(N, V, top, dtype):
    return _bytes("dla_token_logprobs_workspace_size", _LOGPROBS.pack(N, V, top, _code(dtype)))


def token_logprobs_backward(logits, tokens, logprob, lse, dlogprob=None, *, entropy=None, dentropy=None, dlse=None,
                            dlogits=None):
    """The gradient of the logits from those of `token_logprobs`' outputs (None: zero) and the outputs themselves
    (dla_token_logprobs_backward).  dlogits may be the logits, and is otherwise apart from the inputs."""
    desc, dev, f32 = _logits(logits, tokens, 0), logits.device, torch.float32
    N = logits.shape[0]
    for name, t in (("logprob", logprob), ("lse", lse), ("entropy", entropy), ("dlogprob", dlogprob),
                    ("dentropy", dentropy), ("dlse", dlse)):
        _like(t, (N,), f32, dev, name, True)
    if dlogits is None:
        dlogits = _new(logits)
    else:
        _like(dlogits, logits.shape, logits.dtype, dev, "dlogits")
        same = dlogits.data_ptr() == logits.data_ptr() and (N <= 1 or dlogits.stride(0) == logits.stride(0))
        _apart("dlogits", dlogits, None if same else logits, tokens, logprob, lse, entropy, dlogprob, dentropy, dlse)
    _call("dla_token_logprobs_backward", dev, desc, _logit_rows(logits, "logits"), _ptr(tokens), _ptr(logprob),
          _ptr(lse), _ptr(entropy), _ptr(dlogprob), _ptr(dentropy), _ptr(dlse), _logit_rows(dlogits, "dlogits"))
    return dlogits


# ---------------------------------------------------------------------------
# gated feed-forward
# ---------------------------------------------------------------------------
def _ff_rows(t, shape, like, name):
    _like(t, shape, like.dtype, like.device, name)
    _last(t, name)
    return _ROWS.pack(t.data_ptr(), t.stride(0))


def _ff_sizes(x, w_gate, w_up):
    if x.dim() != 2 or w_gate.dim() != 2 or w_gate.shape[1] != x.shape[1]:
        raise ValueError(f"shapes {tuple(x.shape)}, {tuple(w_gate.shape)}: x [N, D] and weights [F, D] are wanted")
    return x.shape[0], x.shape[1], w_gate.shape[0]


def _aligned(x, w_gate, w_up):
    """Whether the library reads these in place: 16-byte aligned rows, one stride of the weights, no wide gaps."""
    def ok(t):
        e = t.element_size()
        return t.data_ptr() % 16 == 0 and (t.shape[0] <= 1 or (t.stride(0) * e % 16 == 0 and t.stride(0) <= 1 << 21))
    return ok(x) and ok(w_gate) and ok(w_up) and (w_gate.shape[0] <= 1 or w_gate.stride(0) == w_up.stride(0))


@functools.lru_cache(maxsize=4096)
def gated_ff_workspace_bytes(N: int, D: int, F: int, dtype=torch.bfloat16, *, backward: bool = False,
                             aligned: bool = True) -> int:
    """Workspace of a forward (or backward) pass.  aligned: rows of x and the weights start at multiples of 16 bytes."""
    return _bytes("dla_gated_ff_workspace_size", _FF.pack(N, D, F, _code(dtype)), int(backward), int(aligned))


def gated_ff(x, w_gate, w_up, *, out=None, want_parts: bool = False, workspace=None):
    """y = silu(x w_gate^T) * (x w_up^T) (dla_gated_ff).  x: [N, D], w_gate and w_up [F, D], last axes contiguous; out
    is apart from them.  Returns (y, parts): the products [2, N, F], float32, that gated_ff_backward needs, or None."""
    N, D, F = _ff_sizes(x, w_gate, w_up)
    dev = x.device
    new = lambda t: _ROWS.pack(t.data_ptr(), F)  # noqa: E731
    if out is None:
        out = x.new_empty((N, F))
        y = new(out)
    else:
        y = _ff_rows(out, (N, F), x, "out")
        _apart("out", out, x, w_gate, w_up)
    parts = x.new_empty((2, N, F), dtype=torch.float32) if want_parts else None
    rows = _ff_rows(x, (N, D), x, "x"), _ff_rows(w_gate, (F, D), x, "w_gate"), _ff_rows(w_up, (F, D), x, "w_up")
    need = gated_ff_workspace_bytes(N, D, F, x.dtype, aligned=_aligned(x, w_gate, w_up))
    workspace, size = _work(workspace, need, dev)
    _call("dla_gated_ff", dev, _FF.pack(N, D, F, _code(x.dtype)), *rows, y,
          *(map(new, parts) if want_parts else (None, None)), _ptr(workspace), size)
    return out, parts


def gated_ff_backward(x, w_gate, w_up, parts, dy, *, workspace=None):
    """Gradients of `gated_ff` (dla_gated_ff_backward) from dy and the forward pass's parts: dx, dw_gate, dw_up, all of
    the inputs' type."""
    N, D, F = _ff_sizes(x, w_gate, w_up)
    dev = x.device
    rows = _ff_rows(x, (N, D), x, "x"), _ff_rows(w_gate, (F, D), x, "w_gate"), _ff_rows(w_up, (F, D), x, "w_up")
    _like(parts, (2, N, F), torch.float32, dev, "parts", True)
    dx, dwg, dwu = x.new_empty((N, D)), x.new_empty((F, D)), x.new_empty((F, D))
    need = gated_ff_workspace_bytes(N, D, F, x.dtype, backward=True, aligned=_aligned(x, w_gate, w_up))
    workspace, size = _work(workspace, need, dev)
    _call("dla_gated_ff_backward", dev, _FF.pack(N, D, F, _code(x.dtype)), *rows,
          _ROWS.pack(parts.data_ptr(), F), _ROWS.pack(parts.data_ptr() + 4 * N * F, F), _ff_rows(dy, (N, F), x, "dy"),
          _ff_rows(dx, (N, D), x, "dx"), _ff_rows(dwg, (F, D), x, "dw_gate"), _ff_rows(dwu, (F, D), x, "dw_up"),
          _ptr(workspace), size)
    return dx, dwg, dwu


# ---------------------------------------------------------------------------
# the same for torch's automatic differentiation, once: the library has no second
# derivatives, and asking for one raises an error
# ---------------------------------------------------------------------------
def _as_rows(t):
    """A gradient as the library reads it: last axis contiguous, no negative strides."""
    return t if t.stride(-1) == 1 or t.shape[-1] <= 1 else t.contiguous()


class ShortConv(torch.autograd.Function):
    """out, last state = ShortConv.apply(x, weight, bias, activation, state, lengths, starts); all but x and weight may
    be None."""

    @staticmethod
    def forward(ctx, x, weight, bias=None, activation="silu", state=None, lengths=None, starts=None):
        x = _as_rows(x)
        out, last = short_conv(x, weight, bias, activation=activation, state=state, lengths=lengths, starts=starts,
                               want_state=True)
        ctx.save_for_backward(x, weight, bias, state, lengths, starts)
        ctx.activation = activation
        ctx.set_materialize_grads(False)
        return out, last

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, dlast):
        x, weight, bias, state, lengths, starts = ctx.saved_tensors
        dout = torch.zeros_like(x) if dout is None else _as_rows(dout.to(x.dtype))
        dx, dw, db, ds = short_conv_backward(x, weight, dout, bias, activation=ctx.activation, state=state,
                                             dstate=None if dlast is None else dlast.to(x.dtype).contiguous(),
                                             lengths=lengths, starts=starts)
        return dx, dw.to(weight.dtype), None if db is None else db.to(bias.dtype), None, ds, None, None


class GatedNorm(torch.autograd.Function):
    """h, y = GatedNorm.apply(x, weight, gate, residual, scale, next_weight, eps): as `gated_norm`, for x [..., D] with a
    weight [D], or [..., G, D] with a weight [G, D].  gate, residual and next_weight may be None; y is None without
    next_weight."""

    @staticmethod
    def _rows(t, weight):
        if t is None:
            return None
        t = t.reshape(-1, *t.shape[-weight.dim():])
        return _as_rows(t)

    @staticmethod
    def forward(ctx, x, weight, gate=None, residual=None, scale=1.0, next_weight=None, eps=1e-6):
        rows = [GatedNorm._rows(t, weight) for t in (x, gate, residual)]
        h, y, rstd, y_rstd = gated_norm(rows[0], weight, *rows[1:], scale=scale, next_weight=next_weight, eps=eps)
        ctx.save_for_backward(*rows, weight, next_weight, rstd, y_rstd)
        ctx.shape, ctx.scale = x.shape, scale
        ctx.set_materialize_grads(False)
        return h.view(x.shape), None if y is None else y.view(x.shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, dh, dy):
        x, gate, residual, weight, next_weight, rstd, y_rstd = ctx.saved_tensors
        rows = lambda t: None if t is None else GatedNorm._rows(t.to(x.dtype), weight)  # noqa: E731
        dh, dy = rows(dh), rows(dy)
        if dh is None:
            dh = torch.zeros_like(x)
        dx, dgate, dres, dw, dw2 = gated_norm_backward(dh, x, weight, rstd, gate, residual, scale=ctx.scale,
                                                       next_weight=next_weight, dy=dy, y_rstd=y_rstd)
        back = lambda t: None if t is None else t.reshape(ctx.shape)  # noqa: E731
        return (back(dx), dw.to(weight.dtype), back(dgate), None if residual is None else back(dres), None,
                None if dw2 is None else dw2.to(next_weight.dtype), None)


class GatedFF(torch.autograd.Function):
    """y = GatedFF.apply(x, w_gate, w_up) for x [..., D]."""

    @staticmethod
    def forward(ctx, x, w_gate, w_up):
        rows = _as_rows(x.reshape(-1, x.shape[-1]))
        y, parts = gated_ff(rows, w_gate, w_up, want_parts=True)
        ctx.save_for_backward(rows, w_gate, w_up, parts)
        ctx.shape = x.shape
        return y.view(*x.shape[:-1], w_gate.shape[0])

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, w_gate, w_up, parts = ctx.saved_tensors
        dy = _as_rows(dy.to(x.dtype).reshape(-1, dy.shape[-1]))
        dx, dwg, dwu = gated_ff_backward(x, w_gate, w_up, parts, dy)
        return dx.view(ctx.shape), dwg, dwu


class TokenLogprobs(torch.autograd.Function):
    """logprob, entropy, lse = TokenLogprobs.apply(logits, tokens) for logits [..., V] and tokens [...]."""

    @staticmethod
    def forward(ctx, logits, tokens):
        rows, tok = _as_rows(logits.reshape(-1, logits.shape[-1])), tokens.reshape(-1).contiguous()
        lp, lse, ent, _, _ = token_logprobs(rows, tok, entropy=True)
        ctx.save_for_backward(rows, tok, lp, lse, ent)
        ctx.shape = logits.shape
        ctx.set_materialize_grads(False)
        return tuple(t.view(tokens.shape) for t in (lp, ent, lse))

    @staticmethod
    @once_differentiable
    def backward(ctx, dlp, dent, dlse):
        rows, tok, lp, lse, ent = ctx.saved_tensors
        flat = lambda t: None if t is None else t.reshape(-1).contiguous()  # noqa: E731
        d = token_logprobs_backward(rows, tok, lp, lse, flat(dlp), entropy=ent, dentropy=flat(dent), dlse=flat(dlse))
        return d.view(ctx.shape), None
