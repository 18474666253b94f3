"""Python binding of libdla's training operators (include/dla_train.h): the
single-state recurrence of the base model with its backward pass, the
root-mean-square norm of the residual stream, and AdamW.  Argument marshalling
only: the work is the library's, torch provides device memory and the current
stream.

Below the calls, the same as differentiable functions (`Recurrence`, `RMSNorm`)
for a model written in torch.
"""
from __future__ import annotations

import ctypes
import functools
import struct
from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import dla
from .dla import DLA_BF16, DLA_F32, _check, _dtype_code

DLA_STATE_FP8 = 2
FP8 = torch.float8_e4m3fn
FP8_BLOCK = 256          # elements per scale of 8-bit optimizer states


# A decode step calls these with little to do on the GPU, so the descriptions of its
# arguments are packed as bytes, which costs a tenth of filling ctypes structures.
_ROWS = struct.Struct("Pqqq")            # dla_rows
_RECURRENCE = struct.Struct("7ifP")      # dla_recurrence_desc
_NORM = struct.Struct("q3if")            # dla_norm_desc
_NORM_ROWS = struct.Struct("Pq")         # dla_norm_rows


class AdamWTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("master", ctypes.c_void_p),
                ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n", ctypes.c_int64), ("weight_decay", ctypes.c_float)]


class AdamWParams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_int64),
                ("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32),
                ("state_format", ctypes.c_int32), ("seed", ctypes.c_uint32),
                ("grad_scale", ctypes.c_void_p)]


@functools.lru_cache(maxsize=None)
def lib():
    """libdla.so with the training entry points declared."""
    L = dla.lib()
    P, S, I = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    L.dla_recurrence_workspace_size.argtypes = [P, I, ctypes.POINTER(S)]
    L.dla_recurrence_forward.argtypes = [P] * 9 + [S, P]
    L.dla_recurrence_backward.argtypes = [P] * 14 + [S, P]
    L.dla_rms_norm.argtypes = [P] * 8
    L.dla_rms_norm_fp8.argtypes = [P] * 8
    L.dla_rms_norm_workspace_size.argtypes = [P, ctypes.POINTER(S)]
    L.dla_rms_norm_backward.argtypes = [P] * 9 + [S, P]
    L.dla_adamw_step.argtypes = [ctypes.POINTER(AdamWTensor), I, ctypes.POINTER(AdamWParams), P]
    for name in dla.EXPORTED:
        if name.startswith(("dla_recurrence", "dla_rms_norm", "dla_adamw")):
            getattr(L, name).restype = ctypes.c_int
    return L


def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device):
    """The current stream's handle, without a Stream object around it where torch has a call for that."""
    if _raw_stream is not None and device.index is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _run(call, device, *args):
    """A library call on the device's current stream.  Kernels go to the calling thread's
    current device, whichever a stream's is."""
    f = getattr(lib(), call)
    if device.index == _current_device():
        status = f(*args, _stream(device))
    else:
        with torch.cuda.device(device):
            status = f(*args, _stream(device))
    _check(status, call)


# ---------------------------------------------------------------------------
# recurrence
# ---------------------------------------------------------------------------
def _rows(t, name):
    """dla_rows of a [B, heads, T, d] tensor, or of a [B, H, T] one."""
    st = t.stride()
    if len(st) == 4 and st[3] != 1 and t.numel():
        raise ValueError(f"{name}: the last axis must be contiguous")
    return _ROWS.pack(t.data_ptr(), st[0], st[1], st[2])


def _desc(B, H, Hk, T, d_k, d_v, dtype, scale=1.0, lengths=None):
    return _RECURRENCE.pack(B, H, Hk, T, d_k, d_v, _dtype_code(dtype), scale,
                            0 if lengths is None else lengths.data_ptr())


@functools.lru_cache(maxsize=4096)
def recurrence_workspace_bytes(B: int, H: int, Hk: int, T: int, d_k: int, d_v: int, dtype, *,
                               backward: bool = False) -> int:
    """Workspace of a forward (or backward) pass; 0 where none is needed."""
    n = ctypes.c_size_t(0)
    _check(lib().dla_recurrence_workspace_size(_desc(B, H, Hk, T, d_k, d_v, dtype), int(backward),
                                               ctypes.byref(n)), "dla_recurrence_workspace_size")
    return int(n.value)


def _sizes(q, k, v, g, lengths):
    """(B, H, Hk, T, d_k, d_v) of a call whose inputs fit each other."""
    B, Hk, T, d_k = q.shape
    _, H, _, d_v = v.shape
    if k.shape != q.shape or v.shape[0] != B or v.shape[2] != T or g.shape != (B, H, T):
        raise ValueError(f"shapes {tuple(q.shape)}, {tuple(k.shape)}, {tuple(v.shape)}, {tuple(g.shape)}")
    dtype, dev = q.dtype, q.device
    if k.dtype != dtype or v.dtype != dtype or g.dtype != torch.float32:
        raise ValueError(f"types {dtype}, {k.dtype}, {v.dtype}, {g.dtype}: one type and float32 gates are wanted")
    if k.device != dev or v.device != dev or g.device != dev:
        raise ValueError("q, k, v and g must be on one device")
    if lengths is not None and (lengths.shape != (B,) or lengths.dtype != torch.int32 or
                                not lengths.is_contiguous() or lengths.device != dev):
        raise ValueError("lengths must be int32 [B], contiguous, on the inputs' device")
    return B, H, Hk, T, d_k, d_v


def _like(t, shape, dtype, device, name, contiguous=False):
    if t is not None and (t.shape != shape or t.dtype != dtype or t.device != device or
                          (contiguous and not t.is_contiguous())):
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, not "
                         f"{'contiguous ' if contiguous else ''}{dtype} {tuple(shape)} on {device}")


def _space(workspace, need, device):
    """A workspace and its size: the caller's, where that is large enough, else a new one."""
    if workspace is not None and (workspace.device != device or not workspace.is_contiguous()):
        raise ValueError(f"workspace must be contiguous on {device}")
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    return workspace, workspace.numel() * workspace.element_size()


def _token_major(B, heads, T, d, dtype, device):
    """[B, heads, T, d], laid out [B][T][heads][d] as projections read it."""
    return torch.empty_strided((B, heads, T, d), (T * heads * d, d, heads * d, 1), dtype=dtype, device=device)


def recurrence(q, k, v, g, *, scale: float = 1.0, state=None, lengths=None, out=None,
               state_out=None, want_state: bool = False, workspace=None):
    """S_t = exp(g_t) S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t (dla_recurrence_forward).
    q, k: [B, Hk, T, d_k]; v: [B, H, T, d_v]; g: [B, H, T] float32, in any layout with the
    last axis of q, k and v contiguous and its rows 16-byte aligned.  state: [B, H, d_k,
    d_v] float32 or None; state_out may be the same tensor.  Returns (out, state_out); out
    is laid out [B][T][H][d_v] unless given."""
    B, H, Hk, T, d_k, d_v = _sizes(q, k, v, g, lengths)
    dtype, dev, f32 = q.dtype, q.device, torch.float32
    _like(state, (B, H, d_k, d_v), f32, dev, "state", True)
    if out is None:
        out = _token_major(B, H, T, d_v, dtype, dev)
    else:
        _like(out, v.shape, dtype, dev, "out")
    if state_out is not None:
        _like(state_out, (B, H, d_k, d_v), f32, dev, "state_out", True)
    elif want_state:
        state_out = torch.empty((B, H, d_k, d_v), dtype=f32, device=dev)
    need, size = recurrence_workspace_bytes(B, H, Hk, T, d_k, d_v, dtype), 0
    if need:
        workspace, size = _space(workspace, need, dev)
    _run("dla_recurrence_forward", dev,
         _desc(B, H, Hk, T, d_k, d_v, dtype, scale, lengths), _rows(q, "q"), _rows(k, "k"), _rows(v, "v"),
         _rows(g, "g"), _ptr(state), _rows(out, "out"), _ptr(state_out), _ptr(workspace) if need else None, size)
    return out, state_out


def recurrence_backward(q, k, v, g, dout, *, scale: float = 1.0, state=None, dstate=None,
                        lengths=None, want_dstate: Optional[bool] = None, workspace=None):
    """Gradients of `recurrence` (dla_recurrence_backward) from those of its outputs, dout
    and dstate (None: zero).  Returns dq, dk, dv, dg, all of the inputs' type, and the
    gradient of `state` (float32; None without one, unless want_dstate)."""
    B, H, Hk, T, d_k, d_v = _sizes(q, k, v, g, lengths)
    dtype, dev, f32 = q.dtype, q.device, torch.float32
    _like(state, (B, H, d_k, d_v), f32, dev, "state", True)
    _like(dstate, (B, H, d_k, d_v), f32, dev, "dstate", True)
    _like(dout, v.shape, dtype, dev, "dout")
    dq = _token_major(B, Hk, T, d_k, dtype, dev)
    dk = _token_major(B, Hk, T, d_k, dtype, dev)
    dv = _token_major(B, H, T, d_v, dtype, dev)
    dg = torch.empty_strided((B, H, T), (T * H, 1, H), dtype=dtype, device=dev)
    ds0 = None
    if state is not None if want_dstate is None else want_dstate:
        ds0 = torch.empty((B, H, d_k, d_v), dtype=f32, device=dev)
    need, size = recurrence_workspace_bytes(B, H, Hk, T, d_k, d_v, dtype, backward=True), 0
    if need:
        workspace, size = _space(workspace, need, dev)
    _run("dla_recurrence_backward", dev,
         _desc(B, H, Hk, T, d_k, d_v, dtype, scale, lengths), _rows(q, "q"), _rows(k, "k"), _rows(v, "v"),
         _rows(g, "g"), _ptr(state), _rows(dout, "dout"), _ptr(dstate), _rows(dq, "dq"), _rows(dk, "dk"),
         _rows(dv, "dv"), _rows(dg, "dg"), _ptr(ds0), _ptr(workspace) if need else None, size)
    return dq, dk, dv, dg, ds0


# ---------------------------------------------------------------------------
# norm
# ---------------------------------------------------------------------------
def _norm_rows(t, like, name):
    if t is None:
        return None
    if t.shape != like.shape or t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, not {like.dtype} "
                         f"{tuple(like.shape)} on {like.device}")
    st = t.stride()
    if st[1] != 1 and t.shape[1] > 1 and t.numel():
        raise ValueError(f"{name}: rows must be contiguous")
    return _NORM_ROWS.pack(t.data_ptr(), st[0])


def _norm_desc(x, weight, eps):
    if x.dim() != 2 or weight.shape != x.shape[1:] or not weight.is_contiguous() or weight.device != x.device:
        raise ValueError(f"shapes {tuple(x.shape)}, {tuple(weight.shape)}: rows [N, D] and a weight [D] are wanted")
    return _NORM.pack(*x.shape, _dtype_code(x.dtype), _dtype_code(weight.dtype), eps)


def _norm_forward(call, x, weight, residual, eps, y, last):
    desc, D = _norm_desc(x, weight, eps), x.shape[1]
    rows = _norm_rows(x, x, "x"), _norm_rows(residual, x, "residual")
    h = None if residual is None else torch.empty_like(residual, memory_format=torch.contiguous_format)
    _run(call, x.device, desc, *rows, weight.data_ptr(),
         None if h is None else _NORM_ROWS.pack(h.data_ptr(), D), _NORM_ROWS.pack(y.data_ptr(), D),
         last.data_ptr())
    return x if h is None else h


def rms_norm(x, weight, residual=None, *, eps: float = 1e-6):
    """h = x + residual, y = weight h / sqrt(mean(h^2) + eps) (dla_rms_norm).  x, residual:
    [N, D].  Returns (y, h, rstd); h is x itself without a residual."""
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    rstd = torch.empty(x.shape[:1], dtype=torch.float32, device=x.device)
    return y, _norm_forward("dla_rms_norm", x, weight, residual, eps, y, rstd), rstd


def rms_norm_fp8(x, weight, residual=None, *, eps: float = 1e-6):
    """The same with y in 8 bits (dla_rms_norm_fp8): returns (y float8_e4m3fn, h, scale),
    y times its row's scale being the norm's output."""
    y = torch.empty(x.shape, dtype=FP8, device=x.device)
    scale = torch.empty(x.shape[:1], dtype=torch.float32, device=x.device)
    return y, _norm_forward("dla_rms_norm_fp8", x, weight, residual, eps, y, scale), scale


@functools.lru_cache(maxsize=4096)
def rms_norm_workspace_bytes(rows: int, D: int, dtype=torch.bfloat16) -> int:
    """Workspace of rms_norm_backward for rows of D values."""
    n = ctypes.c_size_t(0)
    code = _dtype_code(dtype)
    _check(lib().dla_rms_norm_workspace_size(_NORM.pack(rows, D, code, code, 0.0), ctypes.byref(n)),
           "dla_rms_norm_workspace_size")
    return int(n.value)


def rms_norm_backward(dy, h, weight, rstd, dres=None, *, workspace=None):
    """Gradients of rms_norm from dy and dres, those of its outputs y and h (None: zero):
    (dx, which is also the residual's, and dweight in float32)."""
    dev = h.device
    desc = _norm_desc(h, weight, 0.0)
    _like(rstd, h.shape[:1], torch.float32, dev, "rstd", True)
    dx = torch.empty(h.shape, dtype=h.dtype, device=dev)
    dw = torch.empty(h.shape[1:], dtype=torch.float32, device=dev)
    workspace, size = _space(workspace, rms_norm_workspace_bytes(*h.shape, h.dtype), dev)
    _run("dla_rms_norm_backward", dev,
         desc, _norm_rows(dy, h, "dy"), _norm_rows(h, h, "h"), weight.data_ptr(), rstd.data_ptr(),
         _norm_rows(dres, h, "dres"), _norm_rows(dx, h, "dx"), dw.data_ptr(), workspace.data_ptr(), size)
    return dx, dw


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
class AdamW:
    """AdamW over many tensors at once (dla_adamw_step).  `add` names a tensor and its
    buffers, which are kept; `step` updates all of them in place on the current stream.
    Without m and v, `add` makes their states, zeroed, in the given format.  Tensors may
    differ in type; those of a kind go in the same launches.

    Every step works on the memory that the tensors have then: one whose `.data` was
    replaced is followed.  So is a gradient that is `param.grad` when it is added: each step
    takes what `param.grad` then is, so that gradients may be set to None and made anew by
    the next backward pass.  Any other gradient tensor is a buffer for the caller to fill."""

    def __init__(self, states: str = "f32"):
        if states not in ("f32", "fp8"):
            raise ValueError(f"states {states!r}: f32 or fp8")
        self.states = states
        self.kept = []       # the tensors of each entry
        self._groups = {}    # (param, grad type, format, device) -> entries
        self._tensors, self._at = [], []     # what has an address in a description, and which
        self._arrays = None

    def add(self, param, grad, m=None, v=None, *, master=None, m_scale=None, v_scale=None,
            weight_decay: float = 0.0):
        n, dev = param.numel(), param.device
        if m is None and v is None:
            if self.states == "fp8":
                m, v = (torch.zeros(n, dtype=torch.uint8, device=dev).view(FP8) for _ in range(2))
                m_scale, v_scale = (torch.zeros(-(-n // FP8_BLOCK), device=dev) for _ in range(2))
            else:
                m, v = (torch.zeros(n, device=dev) for _ in range(2))
        elif m is None or v is None:
            raise ValueError("m and v come together")
        fp8 = m.dtype == FP8
        if v.dtype != m.dtype or m.dtype not in (torch.float32, FP8):
            raise ValueError(f"states of types {m.dtype}, {v.dtype}")
        if fp8 and (m_scale is None or v_scale is None):
            raise ValueError("8-bit states need their scales")
        key = (_dtype_code(param.dtype), _dtype_code(grad.dtype), DLA_STATE_FP8 if fp8 else DLA_F32, dev)
        tensors = [param, master, grad, m, v] + ([m_scale, v_scale] if fp8 else [None, None])
        self._fit(key, tensors, n)
        own = param.grad if param.is_leaf else None
        follow = own is not None and own.data_ptr() == grad.data_ptr()
        if follow:
            tensors[2] = None       # looked up, and not kept: it may be freed between steps
        self._groups.setdefault(key, []).append((tensors, n, float(weight_decay), follow))
        self.kept.append({"param": param, "master": master, "m": m, "v": v, "m_scale": m_scale,
                          "v_scale": v_scale})
        self._tensors += [t for t in tensors if t is not None]
        self._at += [t.data_ptr() for t in tensors if t is not None]
        self._arrays = None

    @staticmethod
    def _fit(key, tensors, n):
        """Refuses an entry's tensors (in the order of dla_adamw_tensor) that are not its kind's."""
        p, g, fmt, dev = key
        dtypes = {DLA_F32: torch.float32, DLA_BF16: torch.bfloat16}
        state = FP8 if fmt == DLA_STATE_FP8 else torch.float32
        for i, (t, dtype) in enumerate(zip(tensors, (dtypes[p], torch.float32, dtypes[g], state, state,
                                                     torch.float32, torch.float32))):
            size = n if i < 5 else -(-n // FP8_BLOCK)
            if t is not None and (t.numel() != size or t.dtype != dtype or t.device != dev or
                                  not t.is_contiguous() or (size and not t.data_ptr())):
                raise ValueError(f"a buffer of {t.numel()} {t.dtype} on {t.device} where {size} "
                                 f"contiguous {dtype} on {dev} are wanted")

    def _marshal(self):
        """The descriptions of all tensors, and the gradients that every step looks up."""
        self._arrays = [(key, (AdamWTensor * len(es))(*[AdamWTensor(*map(_ptr, e[0]), *e[1:3]) for e in es]))
                        for key, es in self._groups.items()]
        self._followed = [(e[0][0], array[i], key, e[1]) for key, array in self._arrays
                          for i, e in enumerate(self._groups[key]) if e[3]]

    def _refresh(self):
        """Addresses as they are now."""
        at = list(map(torch.Tensor.data_ptr, self._tensors))
        if at != self._at:
            for key, entries in self._groups.items():
                for tensors, n, *_ in entries:
                    self._fit(key, tensors, n)
            self._at, self._arrays = at, None
        if self._arrays is None:
            self._marshal()
        for param, description, key, n in self._followed:
            grad = param.grad
            if grad is None:
                raise ValueError(f"a parameter of shape {tuple(param.shape)} has no gradient")
            self._fit(key, (None, None, grad), n)
            description.grad = grad.data_ptr()

    def step(self, step: int, *, lr: float, betas=(0.9, 0.999), eps: float = 1e-8, seed: int = 0,
             grad_scale=None):
        """The step-th update (from 1).  seed: of 8-bit states' rounding, 0 for nearest.
        grad_scale: a float32 tensor of one element, or None; the step changes nothing where
        it is not finite."""
        self._refresh()
        if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1):
            raise ValueError("grad_scale must be one float32")
        for (p, g, fmt, dev), arr in self._arrays:
            if grad_scale is not None and grad_scale.device != dev:
                raise ValueError(f"grad_scale on {grad_scale.device}, tensors on {dev}")
            args = AdamWParams(lr, betas[0], betas[1], eps, step, p, g, fmt, seed & 0xFFFFFFFF,
                               None if grad_scale is None else grad_scale.data_ptr())
            _run("dla_adamw_step", dev, arr, len(arr), ctypes.byref(args))


# ---------------------------------------------------------------------------
# the same for torch's automatic differentiation, once: the library has no second
# derivatives, and asking for one raises an error
# ---------------------------------------------------------------------------
def _as_rows(t):
    """A gradient as the library reads it: last axis contiguous, rows 16-byte aligned."""
    e = t.element_size()
    if t.stride(-1) != 1 or t.data_ptr() % 16 or any(s * e % 16 for s in t.stride()[:-1]):
        # (contiguous() would hand back a contiguous view at any address)
        return t.clone(memory_format=torch.contiguous_format)
    return t


class Recurrence(torch.autograd.Function):
    """out, last state = Recurrence.apply(q, k, v, g, state, scale, lengths); state and
    lengths may be None."""

    @staticmethod
    def forward(ctx, q, k, v, g, state=None, scale=1.0, lengths=None):
        out, last = recurrence(q, k, v, g, scale=scale, state=state, lengths=lengths, want_state=True)
        ctx.save_for_backward(q, k, v, g, state, lengths)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return out, last

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, dlast):
        q, k, v, g, state, lengths = ctx.saved_tensors
        dout = torch.zeros_like(v) if dout is None else _as_rows(dout.to(v.dtype))
        dq, dk, dv, dg, ds = recurrence_backward(q, k, v, g, dout, scale=ctx.scale, state=state,
                                                 dstate=None if dlast is None else _as_rows(dlast).contiguous(),
                                                 lengths=lengths)
        return dq, dk, dv, dg.to(g.dtype), ds, None, None


def _as_norm_rows(t, D):
    """The rows [N, D] of a tensor as the library reads them: contiguous, and apart."""
    t = t.reshape(-1, D)
    if (D > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < D):
        t = t.contiguous()       # broadcast or transposed
    return t


class RMSNorm(torch.autograd.Function):
    """y, h = RMSNorm.apply(x, residual, weight, eps): h = x + residual, y its norm.
    residual may be None: h is then x."""

    @staticmethod
    def forward(ctx, x, residual, weight, eps=1e-6):
        D = x.shape[-1]
        y, h, rstd = rms_norm(_as_norm_rows(x, D), weight,
                              None if residual is None else _as_norm_rows(residual, D), eps=eps)
        ctx.save_for_backward(h, weight, rstd)
        ctx.shape, ctx.residual = x.shape, residual is not None
        ctx.set_materialize_grads(False)
        return y.view(x.shape), h.view(x.shape) if ctx.residual else x

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh):
        h, weight, rstd = ctx.saved_tensors
        rows = lambda t: _as_norm_rows(t.to(h.dtype), h.shape[1])  # noqa: E731
        dy = torch.zeros_like(h) if dy is None else rows(dy)
        dx, dw = rms_norm_backward(dy, h, weight, rstd, dres=None if dh is None else rows(dh))
        dx = dx.view(ctx.shape)
        return dx, dx if ctx.residual else None, dw.to(weight.dtype), None
