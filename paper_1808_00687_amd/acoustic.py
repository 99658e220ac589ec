"""Binding of the acoustic-model operators of libwfstdec.so (the wfst_am_*
calls in include/wfstdec.h): the layers of a network that scores frames, its
loss against a teacher's top logits, the clipping of its gradients, and its
logits as rows for wfst_decode.

The functions keep the C names and only marshal arguments; every step runs in
the library's HIP kernels.  Operands are torch tensors on one GPU.  A matrix
is two-dimensional; its rows may lie any distance apart (an input whose
columns are not adjacent, or whose rows overlap, is copied first; an output
like that is refused).  Vectors (bias, gain, scales, weights) are float32.
The calls only enqueue, on the ``stream`` that each takes by name (a torch
stream or a raw handle) or else torch's current stream, so they can be captured
into a graph.  Results that a call takes no place for, or is given none for, and
the gradients' workspaces come from torch's allocator on that stream: an 8-bit
norm's scales, a loss and its lse, and all that
wfst_am_linear_backward, wfst_am_gated_backward, wfst_am_norm_backward and
wfst_am_layer_norm_backward return, and wfst_am_clip's norm, always do.  (The C calls allocate nothing.)  Arguments that the library
refuses raise WfstError (WFST_EINVAL) with its message.

Autograd does not follow these calls: an operand that requires a gradient is
refused while gradients are recorded (inside a torch.autograd.Function, under
no_grad and in inference mode they are not), and the gradients are the
``*_backward`` calls'.  A tensor that a call writes counts as changed in place.
"""
from __future__ import annotations

import ctypes as C
import operator
import struct
from itertools import chain, repeat
from typing import Optional, Sequence, Tuple

import torch

from .wfstdec import WFST_OK, WfstError, _lib, wfst_last_error

WFST_F32, WFST_F16, WFST_BF16, WFST_F8E4M3 = range(4)
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
WFST_AM_MAX_TOP = 256

_TYPES = {torch.float32: WFST_F32, torch.float16: WFST_F16, torch.bfloat16: WFST_BF16,
          torch.float8_e4m3fn: WFST_F8E4M3}


class _Matrix(C.Structure):
    _fields_ = [("data", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("row_stride", C.c_int64),
                ("type", C.c_int32), ("reserved", C.c_int32)]


class _LinearArgs(C.Structure):
    _fields_ = [("x", _Matrix), ("w", _Matrix), ("residual", _Matrix), ("pre", _Matrix), ("y", _Matrix),
                ("x_scale", C.c_void_p), ("w_scale", C.c_void_p), ("bias", C.c_void_p),
                ("activation", C.c_int32), ("reserved", C.c_int32)]


class _LinearBackwardArgs(C.Structure):
    _fields_ = [("dy", _Matrix), ("pre", _Matrix), ("x", _Matrix), ("w", _Matrix), ("dx", _Matrix), ("dw", _Matrix),
                ("dbias", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64),
                ("activation", C.c_int32), ("round_dz", C.c_int32)]


class _GatedArgs(C.Structure):
    _fields_ = [("x", _Matrix), ("w", _Matrix), ("pre", _Matrix), ("y", _Matrix), ("x_scale", C.c_void_p),
                ("w_scale", C.c_void_p), ("bias", C.c_void_p), ("activation", C.c_int32), ("reserved", C.c_int32)]


class _GatedBackwardArgs(C.Structure):
    _fields_ = list(_LinearBackwardArgs._fields_)


class _NormArgs(C.Structure):
    _fields_ = [("x", _Matrix), ("residual", _Matrix), ("sum", _Matrix), ("y", _Matrix), ("gain", C.c_void_p),
                ("y_scale", C.c_void_p), ("eps", C.c_float), ("reserved", C.c_int32)]


class _NormBackwardArgs(C.Structure):
    _fields_ = [("dy", _Matrix), ("s", _Matrix), ("dsum", _Matrix), ("dx", _Matrix), ("gain", C.c_void_p),
                ("dgain", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64),
                ("eps", C.c_float), ("reserved", C.c_int32)]


class _LayerNormArgs(C.Structure):
    _fields_ = [("x", _Matrix), ("residual", _Matrix), ("sum", _Matrix), ("y", _Matrix), ("gain", C.c_void_p),
                ("bias", C.c_void_p), ("y_scale", C.c_void_p), ("eps", C.c_float), ("reserved", C.c_int32)]


class _LayerNormBackwardArgs(C.Structure):
    _fields_ = [("dy", _Matrix), ("s", _Matrix), ("dsum", _Matrix), ("dx", _Matrix), ("gain", C.c_void_p),
                ("dgain", C.c_void_p), ("dbias", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_int64), ("eps", C.c_float), ("reserved", C.c_int32)]


class _DistillArgs(C.Structure):
    _fields_ = [("logits", _Matrix), ("top_logit", _Matrix), ("dlogits", _Matrix), ("top_index", C.c_void_p),
                ("weight", C.c_void_p), ("loss", C.c_void_p), ("lse", C.c_void_p), ("temperature", C.c_float),
                ("reserved", C.c_int32)]


class _ClipArgs(C.Structure):
    _fields_ = [("grads", C.c_void_p), ("outs", C.c_void_p), ("count", C.c_int64), ("max_norm", C.c_double),
                ("norm", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]


class _LoglikesArgs(C.Structure):
    _fields_ = [("logits", _Matrix), ("ll", _Matrix), ("log_prior", C.c_void_p), ("scale", C.c_float),
                ("reserved", C.c_int32)]


# Argument structures are packed in one step (a ctypes structure costs more
# per call than a small kernel runs); the layouts are the structures' above.
_M = "Pqqqii"
_PACK = {"linear": struct.Struct(_M * 5 + "PPPii"), "linear_backward": struct.Struct(_M * 6 + "PPqii"),
         "gated": struct.Struct(_M * 4 + "PPPii"), "gated_backward": struct.Struct(_M * 6 + "PPqii"),
         "norm": struct.Struct(_M * 4 + "PPfi"), "norm_backward": struct.Struct(_M * 4 + "PPPqfi"),
         "layer_norm": struct.Struct(_M * 4 + "PPPfi"), "layer_norm_backward": struct.Struct(_M * 4 + "PPPPqfi"),
         "distill": struct.Struct(_M * 3 + "PPPPfi"), "clip": struct.Struct("PPqdPPq"),
         "loglikes": struct.Struct(_M * 2 + "Pfi")}
_NONE = (0, 0, 0, 0, 0, 0)

for _n in ("linear", "linear_backward", "gated", "gated_backward", "norm", "norm_backward", "layer_norm",
           "layer_norm_backward", "distill", "distill_backward", "clip", "loglikes"):
    _f = getattr(_lib, "wfst_am_" + _n)
    _f.argtypes = [C.c_char_p, C.c_void_p]
    _f.restype = C.c_int
for _n in ("linear_backward", "gated_backward", "norm_backward", "layer_norm_backward", "clip"):
    _f = getattr(_lib, "wfst_am_%s_workspace" % _n)
    _f.argtypes = [C.c_char_p, C.POINTER(C.c_int64)]
    _f.restype = C.c_int


_raw_stream = torch._C._cuda_getCurrentRawStream
_written = torch._C._increment_version   # of a sequence of tensors (torch.autograd.graph's wrapper takes as long again)
_DENSE = torch.contiguous_format
_NO_GRAPH = ("%s requires a gradient, which autograd does not get through this call: detach it, or call under "
             "torch.no_grad(); gradients are the *_backward calls'")


def _matrix(t: torch.Tensor, name: str, device: int, keep: Optional[list] = None) -> tuple:
    """A tensor as a wfst_matrix.  An input (``keep`` given) that is not laid
    out as one is copied, and the copy kept until the call is made."""
    code = _TYPES.get(t.dtype)
    if code is None:
        raise TypeError("%s: type %s is not taken" % (name, t.dtype))
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(_NO_GRAPH % name)
    if t.dim() != 2 or t.get_device() != device:
        raise ValueError("%s must be a matrix on the operands' GPU" % name)
    rows, cols = t.shape
    step, inner = t.stride()
    if rows <= 1:
        step = cols
    if (inner != 1 and cols > 1) or step < cols:
        if keep is None:
            raise ValueError("%s must have adjacent columns and rows that do not overlap" % name)
        t = t.contiguous()
        keep.append(t)
        step = cols
    return t.data_ptr(), rows, cols, step, code, 0


def _vector(t: Optional[torch.Tensor], name: str, n: int, device: int, dtype=torch.float32) -> int:
    if t is None:
        return 0
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(_NO_GRAPH % name)
    if t.dtype != dtype or t.get_device() != device or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s must be %d dense %s values on the operands' GPU" % (name, n, str(dtype)[6:]))
    return t.data_ptr()


def _entries(t: torch.Tensor, rows: int, k: int, device: int) -> int:
    if tuple(t.shape) != (rows, k):
        raise ValueError("top_index must be [%d x %d], as top_logit" % (rows, k))
    return _vector(t, "top_index", rows * k, device, torch.int32)


def _device(t: torch.Tensor, name: str) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a torch tensor on a GPU" % name)
    return t.get_device()


class _On:
    """Inside, the operands' device and the given stream are torch's current ones."""

    def __init__(self, device: int, stream):
        if stream is not None and not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(stream), device=device)
        self.guards = [torch.cuda.device(device)] + ([] if stream is None else [torch.cuda.stream(stream)])

    def __enter__(self):
        for g in self.guards:
            g.__enter__()

    def __exit__(self, *exc):
        for g in reversed(self.guards):
            g.__exit__(*exc)


def _here(f):
    """f, which works on the current device and stream, with a ``stream``
    argument and on the device of its first argument (or of that one's first tensor)."""
    operand = f.__code__.co_varnames[0]

    def call(*args, stream=None, **kw):
        first = args[0] if args else kw.get(operand)
        if isinstance(first, (list, tuple)) and first:
            first = first[0]
        if stream is None and (not isinstance(first, torch.Tensor) or not first.is_cuda
                               or first.get_device() == torch._C._cuda_getDevice()):
            return f(*args, **kw)
        with _On(_device(first, operand), stream):
            return f(*args, **kw)

    call.__name__, call.__qualname__, call.__doc__ = f.__name__, f.__qualname__, f.__doc__
    call.__wrapped__ = f
    return call


def _call(name: str, packed: bytes, stream: int) -> None:
    rc = getattr(_lib, name)(packed, stream)
    if rc != WFST_OK:
        raise WfstError(rc, "%s: %s" % (name, wfst_last_error()))


def _bytes_for(name: str, packed: bytes) -> int:
    n = C.c_int64()
    rc = getattr(_lib, name)(packed, C.byref(n))
    if rc != WFST_OK:
        raise WfstError(rc, "%s: %s" % (name, wfst_last_error()))
    return n.value


def _activation(name: str) -> int:
    if name not in ACTIVATIONS:
        raise ValueError("activation must be one of %s" % ", ".join(ACTIVATIONS))
    return ACTIVATIONS[name]


@_here
def wfst_am_linear(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, *,
                   activation: str = "none", residual: Optional[torch.Tensor] = None,
                   x_scale: Optional[torch.Tensor] = None, w_scale: Optional[torch.Tensor] = None,
                   pre: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                   out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """act(x w^T [* x_scale w_scale] + bias) + residual: x [M x K], w [N x K]
    -> [M x N] (wfst_am_linear).  ``out_dtype``: that of ``out``, else the
    residual's, else x's (bfloat16 for 8-bit x).  ``pre`` receives the value
    before the activation, for the gradient; ``residual`` may be ``out``."""
    d, keep = _device(x, "x"), []
    mx, mw = _matrix(x, "x", d, keep), _matrix(w, "w", d, keep)
    given = out is not None
    if not given:
        dt = out_dtype or (residual.dtype if residual is not None else
                           torch.bfloat16 if x.dtype == torch.float8_e4m3fn else x.dtype)
        out = x.new_empty((mx[1], mw[1]), dtype=dt)
    elif out_dtype is not None and out_dtype != out.dtype:
        raise ValueError("out_dtype differs from out's")
    _call("wfst_am_linear", _PACK["linear"].pack(
        *mx, *mw, *(_NONE if residual is None else _matrix(residual, "residual", d, keep)),
        *(_NONE if pre is None else _matrix(pre, "pre", d)), *_matrix(out, "out", d),
        _vector(x_scale, "x_scale", mx[1], d), _vector(w_scale, "w_scale", mw[1], d),
        _vector(bias, "bias", mw[1], d), _activation(activation), 0), _raw_stream(d))
    if pre is not None:
        _written((pre,))
    if given:
        _written((out,))
    return out


@_here
def wfst_am_linear_backward(dy: torch.Tensor, x: Optional[torch.Tensor], w: Optional[torch.Tensor], *,
                            activation: str = "none", pre: Optional[torch.Tensor] = None,
                            bias_gradient: bool = True, weight_dtype: Optional[torch.dtype] = None,
                            round_dz: bool = False) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(dx, dw, dbias) of wfst_am_linear with a 16-bit x (the residual's
    gradient is dy).  ``w`` None leaves out dx, ``x`` None dw.
    ``weight_dtype``: dw's type, dy's by default.  ``round_dz``: dx and dw from
    a silu's or gelu's dz rounded to 16 bits, faster, where two 16-bit values
    hold it otherwise."""
    d, keep = _device(dy, "dy"), []
    act, rounded = _activation(activation), int(bool(round_dz))
    mdy = _matrix(dy, "dy", d, keep)
    if act and pre is None:
        raise ValueError("the activation's gradient needs pre")
    mpre = _matrix(pre, "pre", d, keep) if act else _NONE
    mx = _NONE if x is None else _matrix(x, "x", d, keep)
    mw = _NONE if w is None else _matrix(w, "w", d, keep)
    dx = None if w is None else dy.new_empty((mdy[1], mw[2]))
    dw = None if x is None else dy.new_empty((mdy[2], mx[2]), dtype=weight_dtype or dy.dtype)
    db = dy.new_empty(mdy[2], dtype=torch.float32) if bias_gradient else None
    head = (*mdy, *mpre, *mx, *mw, *(_NONE if dx is None else _matrix(dx, "dx", d)),
            *(_NONE if dw is None else _matrix(dw, "dw", d)), 0 if db is None else db.data_ptr())
    pack = _PACK["linear_backward"].pack
    need = _bytes_for("wfst_am_linear_backward_workspace", pack(*head, 0, 0, act, rounded))
    work = dy.new_empty(need, dtype=torch.uint8) if need else None
    _call("wfst_am_linear_backward", pack(*head, work.data_ptr() if need else 0, need, act, rounded), _raw_stream(d))
    return dx, dw, db


@_here
def wfst_am_gated(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, *,
                  activation: str = "silu", x_scale: Optional[torch.Tensor] = None,
                  w_scale: Optional[torch.Tensor] = None, pre: Optional[torch.Tensor] = None,
                  out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """act(gate) * value, both of z = x w^T [* x_scale w_scale] + bias: x [M x K],
    w [2 N x K], the gates' rows and then the values' -> [M x N] (wfst_am_gated).
    ``out_dtype``: that of ``out``, else x's (bfloat16 for 8-bit x).  ``pre``
    [M x 2 N] receives z, for the gradient."""
    d, keep = _device(x, "x"), []
    mx, mw = _matrix(x, "x", d, keep), _matrix(w, "w", d, keep)
    if mw[1] % 2:
        raise ValueError("w must have a row for each gate and one for each value")
    given = out is not None
    if not given:
        dt = out_dtype or (torch.bfloat16 if x.dtype == torch.float8_e4m3fn else x.dtype)
        out = x.new_empty((mx[1], mw[1] // 2), dtype=dt)
    elif out_dtype is not None and out_dtype != out.dtype:
        raise ValueError("out_dtype differs from out's")
    _call("wfst_am_gated", _PACK["gated"].pack(
        *mx, *mw, *(_NONE if pre is None else _matrix(pre, "pre", d)), *_matrix(out, "out", d),
        _vector(x_scale, "x_scale", mx[1], d), _vector(w_scale, "w_scale", mw[1], d),
        _vector(bias, "bias", mw[1], d), _activation(activation), 0), _raw_stream(d))
    if pre is not None:
        _written((pre,))
    if given:
        _written((out,))
    return out


@_here
def wfst_am_gated_backward(dy: torch.Tensor, pre: torch.Tensor, x: Optional[torch.Tensor], w: Optional[torch.Tensor], *,
                           activation: str = "silu", bias_gradient: bool = True,
                           weight_dtype: Optional[torch.dtype] = None, round_dz: bool = False
                           ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(dx, dw, dbias) of wfst_am_gated with a 16-bit x, from its ``pre``.  ``w``
    None leaves out dx, ``x`` None dw.  ``weight_dtype``: dw's type, dy's by
    default.  ``round_dz``: dx and dw from a dz rounded to 16 bits, faster, where
    two 16-bit values hold it otherwise."""
    d, keep = _device(dy, "dy"), []
    act, rounded = _activation(activation), int(bool(round_dz))
    mdy, mpre = _matrix(dy, "dy", d, keep), _matrix(pre, "pre", d, keep)
    mx = _NONE if x is None else _matrix(x, "x", d, keep)
    mw = _NONE if w is None else _matrix(w, "w", d, keep)
    dx = None if w is None else dy.new_empty((mdy[1], mw[2]))
    dw = None if x is None else dy.new_empty((2 * mdy[2], mx[2]), dtype=weight_dtype or dy.dtype)
    db = dy.new_empty(2 * mdy[2], dtype=torch.float32) if bias_gradient else None
    head = (*mdy, *mpre, *mx, *mw, *(_NONE if dx is None else _matrix(dx, "dx", d)),
            *(_NONE if dw is None else _matrix(dw, "dw", d)), 0 if db is None else db.data_ptr())
    pack = _PACK["gated_backward"].pack
    need = _bytes_for("wfst_am_gated_backward_workspace", pack(*head, 0, 0, act, rounded))
    work = dy.new_empty(need, dtype=torch.uint8) if need else None
    _call("wfst_am_gated_backward", pack(*head, work.data_ptr() if need else 0, need, act, rounded), _raw_stream(d))
    return dx, dw, db


@_here
def wfst_am_norm(x: torch.Tensor, gain: Optional[torch.Tensor] = None, *, residual: Optional[torch.Tensor] = None,
                 eps: float = 1e-6, out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
                 sum_out: Optional[torch.Tensor] = None
                 ) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(y, y_scale, sum): the root-mean-square norm of x + residual times
    ``gain`` (wfst_am_norm).  With ``out_dtype`` torch.float8_e4m3fn, y_scale
    [M] is what the rows of y stand for; else None.  ``sum`` is x + residual
    (None without a residual), in ``sum_out`` where given, which may be x or
    residual."""
    d, keep = _device(x, "x"), []
    mx = _matrix(x, "x", d, keep)
    mr = _NONE if residual is None else _matrix(residual, "residual", d, keep)
    given = [t for t in (out, sum_out) if t is not None]
    if out is None:
        out = torch.empty_like(x, dtype=out_dtype or x.dtype, memory_format=_DENSE)
    elif out_dtype is not None and out_dtype != out.dtype:
        raise ValueError("out_dtype differs from out's")
    if sum_out is None and residual is not None:
        sum_out = torch.empty_like(x, memory_format=_DENSE)
    scale = x.new_empty(mx[1], dtype=torch.float32) if out.dtype == torch.float8_e4m3fn else None
    _call("wfst_am_norm", _PACK["norm"].pack(
        *mx, *mr, *(_NONE if sum_out is None else _matrix(sum_out, "sum_out", d)), *_matrix(out, "out", d),
        _vector(gain, "gain", mx[2], d), 0 if scale is None else scale.data_ptr(), eps, 0), _raw_stream(d))
    if given:
        _written(given)
    return out, scale, sum_out


@_here
def wfst_am_norm_backward(dy: torch.Tensor, s: torch.Tensor, gain: Optional[torch.Tensor] = None, *,
                          dsum: Optional[torch.Tensor] = None, eps: float = 1e-6, gain_gradient: bool = True
                          ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(dx, dgain) of wfst_am_norm at its sum ``s`` (x itself without a
    residual); dx is the gradient of x and of residual.  ``dsum``: the
    gradient that reaches the sum past the norm."""
    d, keep = _device(dy, "dy"), []
    mdy, ms = _matrix(dy, "dy", d, keep), _matrix(s, "s", d, keep)
    dx = torch.empty_like(s, memory_format=_DENSE)
    dg = s.new_empty(ms[2], dtype=torch.float32) if gain_gradient else None
    head = (*mdy, *ms, *(_NONE if dsum is None else _matrix(dsum, "dsum", d, keep)), *_matrix(dx, "dx", d),
            _vector(gain, "gain", ms[2], d), 0 if dg is None else dg.data_ptr())
    pack = _PACK["norm_backward"].pack
    need = _bytes_for("wfst_am_norm_backward_workspace", pack(*head, 0, 0, eps, 0))
    work = s.new_empty(need, dtype=torch.uint8) if need else None
    _call("wfst_am_norm_backward", pack(*head, work.data_ptr() if need else 0, need, eps, 0), _raw_stream(d))
    return dx, dg


@_here
def wfst_am_layer_norm(x: torch.Tensor, gain: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *,
                       residual: Optional[torch.Tensor] = None, eps: float = 1e-5,
                       out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
                       sum_out: Optional[torch.Tensor] = None
                       ) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(y, y_scale, sum): the layer norm of x + residual, times ``gain`` plus
    ``bias`` (wfst_am_layer_norm).  With ``out_dtype`` torch.float8_e4m3fn,
    y_scale [M] is what the rows of y stand for; else None.  ``sum`` is
    x + residual (None without a residual), in ``sum_out`` where given, which
    may be x or residual."""
    d, keep = _device(x, "x"), []
    mx = _matrix(x, "x", d, keep)
    mr = _NONE if residual is None else _matrix(residual, "residual", d, keep)
    given = [t for t in (out, sum_out) if t is not None]
    if out is None:
        out = torch.empty_like(x, dtype=out_dtype or x.dtype, memory_format=_DENSE)
    elif out_dtype is not None and out_dtype != out.dtype:
        raise ValueError("out_dtype differs from out's")
    if sum_out is None and residual is not None:
        sum_out = torch.empty_like(x, memory_format=_DENSE)
    scale = x.new_empty(mx[1], dtype=torch.float32) if out.dtype == torch.float8_e4m3fn else None
    _call("wfst_am_layer_norm", _PACK["layer_norm"].pack(
        *mx, *mr, *(_NONE if sum_out is None else _matrix(sum_out, "sum_out", d)), *_matrix(out, "out", d),
        _vector(gain, "gain", mx[2], d), _vector(bias, "bias", mx[2], d), 0 if scale is None else scale.data_ptr(),
        eps, 0), _raw_stream(d))
    if given:
        _written(given)
    return out, scale, sum_out


@_here
def wfst_am_layer_norm_backward(dy: torch.Tensor, s: torch.Tensor, gain: Optional[torch.Tensor] = None, *,
                                dsum: Optional[torch.Tensor] = None, eps: float = 1e-5, gain_gradient: bool = True,
                                bias_gradient: bool = True
                                ) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(dx, dgain, dbias) of wfst_am_layer_norm at its sum ``s`` (x itself
    without a residual); dx is the gradient of x and of residual.  ``dsum``:
    the gradient that reaches the sum past the norm."""
    d, keep = _device(dy, "dy"), []
    mdy, ms = _matrix(dy, "dy", d, keep), _matrix(s, "s", d, keep)
    dx = torch.empty_like(s, memory_format=_DENSE)
    dg = s.new_empty(ms[2], dtype=torch.float32) if gain_gradient else None
    db = s.new_empty(ms[2], dtype=torch.float32) if bias_gradient else None
    head = (*mdy, *ms, *(_NONE if dsum is None else _matrix(dsum, "dsum", d, keep)), *_matrix(dx, "dx", d),
            _vector(gain, "gain", ms[2], d), 0 if dg is None else dg.data_ptr(), 0 if db is None else db.data_ptr())
    pack = _PACK["layer_norm_backward"].pack
    need = _bytes_for("wfst_am_layer_norm_backward_workspace", pack(*head, 0, 0, eps, 0))
    work = s.new_empty(need, dtype=torch.uint8) if need else None
    _call("wfst_am_layer_norm_backward", pack(*head, work.data_ptr() if need else 0, need, eps, 0), _raw_stream(d))
    return dx, dg, db


@_here
def wfst_am_distill(logits: torch.Tensor, top_index: torch.Tensor, top_logit: torch.Tensor, *,
                    temperature: float = 1.0, weight: Optional[torch.Tensor] = None, gradient: bool = False,
                    dlogits: Optional[torch.Tensor] = None
                    ) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """(loss [M], lse [M], dlogits): the loss of the student's logits [M x L]
    against the teacher's top entries (top_index [M x k] int32, top_logit
    [M x k]), and with ``gradient`` (or a tensor for it in ``dlogits``, which
    may be logits) the gradient of the summed loss (wfst_am_distill)."""
    d, keep = _device(logits, "logits"), []
    mx, mt = _matrix(logits, "logits", d, keep), _matrix(top_logit, "top_logit", d, keep)
    loss = logits.new_empty(mx[1], dtype=torch.float32)
    lse = torch.empty_like(loss)
    given = dlogits is not None
    if not given and gradient:
        dlogits = torch.empty_like(logits, memory_format=_DENSE)
    _call("wfst_am_distill", _PACK["distill"].pack(
        *mx, *mt, *(_NONE if dlogits is None else _matrix(dlogits, "dlogits", d)),
        _entries(top_index, mt[1], mt[2], d), _vector(weight, "weight", mx[1], d),
        loss.data_ptr(), lse.data_ptr(), temperature, 0), _raw_stream(d))
    if given:
        _written((dlogits,))
    return loss, lse, dlogits


@_here
def wfst_am_distill_backward(logits: torch.Tensor, top_index: torch.Tensor, top_logit: torch.Tensor,
                             lse: torch.Tensor, *, temperature: float = 1.0, weight: Optional[torch.Tensor] = None,
                             dlogits: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dlogits alone, from the forward call's lse (wfst_am_distill_backward);
    ``weight``: the gradient that reaches each row's loss, times the forward
    call's weight."""
    d, keep = _device(logits, "logits"), []
    mx, mt = _matrix(logits, "logits", d, keep), _matrix(top_logit, "top_logit", d, keep)
    given = dlogits is not None
    if not given:
        dlogits = torch.empty_like(logits, memory_format=_DENSE)
    _call("wfst_am_distill_backward", _PACK["distill"].pack(
        *mx, *mt, *_matrix(dlogits, "dlogits", d),
        _entries(top_index, mt[1], mt[2], d), _vector(weight, "weight", mx[1], d),
        0, _vector(lse, "lse", mx[1], d), temperature, 0), _raw_stream(d))
    if given:
        _written((dlogits,))
    return dlogits


_numel, _dense, _place, _gpu = (torch.Tensor.numel, torch.Tensor.is_contiguous, torch.Tensor.data_ptr,
                                torch.Tensor.get_device)
_dtype, _grad = operator.attrgetter("dtype"), operator.attrgetter("requires_grad")


def _tensors(ts, name: str, device: int, keep: Optional[list] = None) -> list:
    """Tensors of any shape as wfst_matrix fields, one after the other.  A dense one is a single row (rows of its
    last dimension where one would be too long); one that is not has to be a matrix (or is copied, if ``keep`` is
    given)."""
    codes = list(map(_TYPES.get, map(_dtype, ts)))   # (whole lists at a time: a model has hundreds)
    if None in codes:
        raise TypeError("%s: type %s is not taken" % (name, ts[codes.index(None)].dtype))
    if torch.is_grad_enabled() and any(map(_grad, ts)):
        raise ValueError(_NO_GRAPH % name)
    if set(map(_gpu, ts)) != {device}:
        raise ValueError("%s must be on one GPU" % name)
    counts = list(map(_numel, ts))
    if all(map(_dense, ts)) and min(counts) > 0 and max(counts) < 1 << 31:
        return list(chain.from_iterable(zip(map(_place, ts), repeat(1), counts, counts, codes, repeat(0))))
    flat = []
    for t, code, n in zip(ts, codes, counts):
        if n and not t.is_contiguous():
            if t.dim() == 2 or keep is None:
                flat.extend(_matrix(t, name, device, keep))
                continue
            t = t.contiguous()
            keep.append(t)
        cols = n if n < 1 << 31 else t.shape[-1]
        flat.extend((t.data_ptr(), n // cols, cols, cols, code, 0) if n else (0, 0, 1, 1, code, 0))
    return flat


def _pair(a: list, b: list) -> None:
    """The fields of pairs of tensors, where some differ in rows or columns: a single row beside a matrix of as many
    values becomes one, too."""
    for i in range(1, len(a), 6):
        if a[i] != b[i]:
            few, many = (a, b) if a[i] == 1 else (b, a)
            if few[i] == 1 and few[i + 1] == many[i] * many[i + 1]:
                few[i], few[i + 1], few[i + 2] = many[i], many[i + 1], many[i + 1]


@_here
def wfst_am_clip(grads: Sequence[torch.Tensor], max_norm: float, *, out: Optional[Sequence[torch.Tensor]] = None
                 ) -> Tuple[Sequence[torch.Tensor], torch.Tensor]:
    """(out, norm): the tensors times what keeps the norm of all of them within
    ``max_norm`` (infinity: as they are), in ``out`` (a tensor of the same type
    and number of values for each, in the same order) or else in place; ``norm``
    [1] is that before the clipping (wfst_am_clip).  Tensors that are not dense
    have to be matrices; a parameter's gradient may be of any shape, its last
    dimension below 2^31."""
    if not isinstance(grads, (list, tuple)) or not grads:
        raise TypeError("grads must be a list of one tensor or more")
    d, n, keep = _device(grads[0], "grads"), len(grads), []
    layout = _M * n
    if out is None:
        to = grads
        read = written = struct.pack(layout, *_tensors(grads, "grads", d))
    else:
        to = out
        if not isinstance(out, (list, tuple)) or len(out) != n:
            raise ValueError("out must be a list of as many tensors as grads")
        values, places = _tensors(grads, "grads", d, keep), _tensors(out, "out", d)
        if values[1::6] != places[1::6] or values[2::6] != places[2::6]:
            _pair(values, places)
        read, written = struct.pack(layout, *values), struct.pack(layout, *places)
    first = grads[0]
    norm = first.new_empty(1, dtype=torch.float32)
    at = C.cast(C.c_char_p(read), C.c_void_p).value
    head = (at, 0 if out is None else C.cast(C.c_char_p(written), C.c_void_p).value, n, max_norm, norm.data_ptr())
    pack = _PACK["clip"].pack
    need = _bytes_for("wfst_am_clip_workspace", pack(*head, 0, 0))
    work = first.new_empty(need, dtype=torch.uint8)
    _call("wfst_am_clip", pack(*head, work.data_ptr(), need), _raw_stream(d))
    _written(tuple(to))
    return to, norm


@_here
def wfst_am_loglikes(logits: torch.Tensor, log_prior: Optional[torch.Tensor] = None, *, scale: float = 1.0,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scale * (log softmax(logits) - log_prior), float32 [M x L]: rows for
    wfst_decode (wfst_am_loglikes)."""
    d, keep = _device(logits, "logits"), []
    mx = _matrix(logits, "logits", d, keep)
    given = out is not None
    if not given:
        out = torch.empty_like(logits, dtype=torch.float32, memory_format=_DENSE)
    _call("wfst_am_loglikes", _PACK["loglikes"].pack(
        *mx, *_matrix(out, "out", d), _vector(log_prior, "log_prior", mx[2], d), scale, 0), _raw_stream(d))
    if given:
        _written((out,))
    return out
