"""Training operators of include/fa.h: layer norm with its gradient, activation checkpoints in 8 bits,
and the backward passes that read such checkpoints (layer norm, GELU, weight of a linear layer).

As in the rest of the binding a function marshals its arguments and calls the entry point of the same
name.  Activations are tensors of shape (..., cols), float32 or bfloat16, whose last dimension is
dense and whose leading dimensions collapse into rows of one stride.  Parameter gradients may be views
into a worker's row of the gradient matrix: contiguous, float32 or bfloat16, no alignment beyond their
element's.  Where a gradient argument is None a float32 tensor (or one of its partner's type) is
allocated; False leaves it out.

With `stream` given, whatever a function allocates itself comes from that stream's pool and the work is
enqueued there; inputs written on another stream have to be ordered before it by the caller.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools

import torch

from . import FA_BF16, FA_F32, _check, _d, _i, _lib, _ll, _sz, _vp  # noqa: F401

GELU_APPROXIMATE = {"erf": 0, "tanh": 1}

_f = ctypes.c_float
_lib.fa_checkpoint8_bytes.argtypes = [_ll, _ll, ctypes.POINTER(_sz)]
_lib.fa_checkpoint8_store.argtypes = [_vp, _ll, _i, _ll, _ll, _vp, _vp]
_lib.fa_checkpoint8_load.argtypes = [_vp, _i, _ll, _ll, _vp, _ll, _vp]
_lib.fa_layer_norm_forward.argtypes = [_vp, _ll, _vp, _ll, _i, _ll, _ll, _vp, _vp, _i, _f, _vp, _ll, _vp, _ll, _vp, _vp,
                                       _vp, _vp, _vp]
_lib.fa_layer_norm_backward_workspace_bytes.argtypes = [_ll, _ll, ctypes.POINTER(_sz)]
_lib.fa_layer_norm_backward.argtypes = [_vp, _ll, _vp, _ll, _vp, _i, _ll, _ll, _vp, _i, _vp, _vp, _vp, _ll, _vp, _ll, _vp,
                                        _vp, _i, _vp, _sz, _vp]
_lib.fa_gelu_forward.argtypes = [_vp, _ll, _i, _ll, _ll, _vp, _i, _i, _vp, _ll, _vp, _vp, _vp]
_lib.fa_gelu_backward_workspace_bytes.argtypes = [_ll, _ll, ctypes.POINTER(_sz)]
_lib.fa_gelu_backward.argtypes = [_vp, _ll, _vp, _ll, _vp, _i, _vp, _i, _ll, _ll, _i, _vp, _ll, _vp, _i, _vp, _sz, _vp]
_lib.fa_linear_weight_grad_workspace_bytes.argtypes = [_ll, _ll, _ll, _i, ctypes.POINTER(_sz)]
_lib.fa_linear_weight_grad.argtypes = [_vp, _ll, _i, _ll, _ll, _vp, _ll, _vp, _vp, _i, _vp, _sz, _vp]
for _name in ("fa_checkpoint8_bytes", "fa_checkpoint8_store", "fa_checkpoint8_load", "fa_layer_norm_forward",
              "fa_layer_norm_backward_workspace_bytes", "fa_layer_norm_backward", "fa_gelu_forward",
              "fa_gelu_backward_workspace_bytes", "fa_gelu_backward", "fa_linear_weight_grad_workspace_bytes",
              "fa_linear_weight_grad"):
    getattr(_lib, _name).restype = _i

_CODES = {torch.float32: FA_F32, torch.bfloat16: FA_BF16}
_HERE = contextlib.nullcontext()


# ---------------------------------------------------------------------------- arguments

def _code(t, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    return code


def _row_stride(t, name):
    """Stride of the rows that the leading dimensions of t collapse into."""
    if t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1):
        return t.stride(0)
    if t.stride(-1) != 1 and t.shape[-1] != 1:
        raise ValueError(f"{name} must be dense along its last dimension")
    ld, span = None, 1
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if ld is None:
            ld = stride
        elif stride != ld * span:
            raise ValueError(f"the leading dimensions of {name} must collapse into rows of one stride")
        span *= size
    return t.shape[-1] if ld is None else ld


def _matrix(t, name, like=None):
    """(pointer, row stride, rows, cols) of an activation; `like`: (rows, cols, dtype, device) it has to share."""
    _code(t, name)
    if t.dim() < 1 or t.shape[-1] < 1:
        raise ValueError(f"{name} must have a last dimension of at least one element")
    cols = t.shape[-1]
    rows = t.numel() // cols
    if like is not None and (rows, cols, t.dtype) != like[:3]:
        raise ValueError(f"{name} must have {like[0]} rows of {like[1]} elements of {like[2]}, got {rows} of {cols} of {t.dtype}")
    ld = cols if t.is_contiguous() else _row_stride(t, name)
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if like is not None and t.device != like[3]:
        raise ValueError(f"{name} is on {t.device}, the call runs on {like[3]}")
    return t.data_ptr(), ld, rows, cols


def _opt_matrix(t, name, like):
    return (None, 0) if t is None else _matrix(t, name, like)[:2]


def _vector(t, numel, name, device, dtype=None):
    """Pointer of a contiguous tensor of exactly `numel` elements, of `dtype` or of either float type."""
    if dtype is None:
        _code(t, name)
    elif not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    elif t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() != numel:
        raise ValueError(f"{name} must have {numel} elements, got {t.numel()}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the call runs on {device}")
    return t.data_ptr()


def _params(first, second, numel, names, device):
    """Pointers and common type code of two optional parameter vectors."""
    given = [t for t in (first, second) if t is not None]
    ptrs = [None if t is None else _vector(t, numel, n, device) for t, n in zip((first, second), names)]
    if len(given) == 2 and given[0].dtype != given[1].dtype:
        raise ValueError(f"{names[0]} and {names[1]} must have the same dtype")
    return ptrs[0], ptrs[1], _CODES[given[0].dtype] if given else FA_F32


def _buffer(t, nbytes, name, device):
    """Pointer of a byte buffer (checkpoint, workspace) of at least nbytes."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() * t.element_size() < nbytes:
        raise ValueError(f"{name} must have at least {nbytes} bytes, got {t.numel() * t.element_size()}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the call runs on {device}")
    return t.data_ptr()


def _opt_checkpoint(t, rows, cols, name, device):
    return None if t is None else _buffer(t, fa_checkpoint8_bytes(rows, cols), name, device)


def _grads(first, second, shapes, names, device):
    """Tensors for two parameter gradients (see the module's docstring for None and False)."""
    given = [t for t in (first, second) if isinstance(t, torch.Tensor)]
    for t, n in zip((first, second), names):
        if t is not None and t is not False and not isinstance(t, torch.Tensor):
            raise TypeError(f"{n} must be a torch tensor, None or False")
    dtype = given[0].dtype if given else torch.float32
    if len(given) == 2 and given[1].dtype != dtype:
        raise ValueError(f"{names[0]} and {names[1]} must have the same dtype")
    out, ptrs = [], []
    for t, shape, n in zip((first, second), shapes, names):
        if t is False:
            out.append(None)
            ptrs.append(None)
            continue
        if t is None:
            t = torch.empty(shape, dtype=dtype, device=device)
        numel = 1
        for k in shape:
            numel *= k
        out.append(t)
        ptrs.append(_vector(t, numel, n, device))
    if dtype not in _CODES:
        raise TypeError(f"{names[0]} and {names[1]} must be float32 or bfloat16, got {dtype}")
    return out, ptrs, _CODES[dtype]


def _on(device, stream):
    """Context in which a call allocates and launches."""
    if stream is None:
        return _HERE if torch.cuda.current_device() == device.index else torch.cuda.device(device)
    if stream.device != device:
        raise ValueError(f"stream belongs to {stream.device}, the tensors are on {device}")
    return torch.cuda.stream(stream)


def _handle(device):
    return torch.cuda.current_stream(device).cuda_stream


def _workspace(ws, nbytes, device):
    if ws is None:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        return ws, ws.data_ptr(), nbytes
    return ws, _buffer(ws, nbytes, "ws", device), ws.numel() * ws.element_size()


def _approximate(name):
    if name not in GELU_APPROXIMATE:
        raise ValueError(f"approximate must be one of {sorted(GELU_APPROXIMATE)}, got {name!r}")
    return GELU_APPROXIMATE[name]


@functools.lru_cache(maxsize=4096)
def _bytes_of(what, *shape):
    out = _sz(0)
    _check(getattr(_lib, what)(*shape, ctypes.byref(out)), what)
    return int(out.value)


# ---------------------------------------------------------------------------- operators

def fa_checkpoint8_bytes(rows: int, cols: int) -> int:
    return _bytes_of("fa_checkpoint8_bytes", rows, cols)


def new_checkpoint8(rows: int, cols: int, device) -> torch.Tensor:
    """An uninitialised checkpoint buffer for rows x cols activations."""
    return torch.empty(fa_checkpoint8_bytes(rows, cols), dtype=torch.uint8, device=device)


def fa_checkpoint8_store(x, ck=None, stream=None):
    """Checkpoint of the activations x; returns its buffer."""
    xp, ldx, rows, cols = _matrix(x, "x")
    dev = x.device
    with _on(dev, stream):
        ck = new_checkpoint8(rows, cols, dev) if ck is None else ck
        cp = _opt_checkpoint(ck, rows, cols, "ck", dev)
        _check(_lib.fa_checkpoint8_store(xp, ldx, _CODES[x.dtype], rows, cols, cp, _handle(dev)), "fa_checkpoint8_store")
    return ck


def fa_checkpoint8_load(ck, rows, cols, out=None, dtype=torch.bfloat16, stream=None):
    """The rows x cols activations that ck holds, as `out` or a new tensor of `dtype`."""
    if not isinstance(ck, torch.Tensor):
        raise TypeError("ck must be a torch tensor")
    dev = ck.device
    cp = _buffer(ck, fa_checkpoint8_bytes(rows, cols), "ck", dev)
    with _on(dev, stream):
        out = torch.empty((rows, cols), dtype=dtype, device=dev) if out is None else out
        op, ldo, _, _ = _matrix(out, "out", (rows, cols, out.dtype, dev))
        _check(_lib.fa_checkpoint8_load(cp, _CODES[out.dtype], rows, cols, op, ldo, _handle(dev)), "fa_checkpoint8_load")
    return out


def fa_layer_norm_forward(x, weight=None, bias=None, eps=1e-5, residual=None, y=None, sum_out=None, mean=None, rstd=None,
                          ck_sum=None, ck_y=None, stream=None):
    """Layer norm of s = x + residual; returns (y, mean, rstd, s).

    Without a residual s is x itself (sum_out None).  ck_sum / ck_y: buffers of new_checkpoint8() that
    receive the checkpoints of s and of y.
    """
    xp, ldx, rows, cols = _matrix(x, "x")
    dev = x.device
    like = (rows, cols, x.dtype, dev)
    rp, ldr = _opt_matrix(residual, "residual", like)
    wp, bp, pcode = _params(weight, bias, cols, ("weight", "bias"), dev)
    with _on(dev, stream):
        y = torch.empty(x.shape, dtype=x.dtype, device=dev) if y is None else y
        if sum_out is None and residual is not None:
            sum_out = torch.empty(x.shape, dtype=x.dtype, device=dev)
        mean = torch.empty(rows, dtype=torch.float32, device=dev) if mean is None else mean
        rstd = torch.empty(rows, dtype=torch.float32, device=dev) if rstd is None else rstd
        yp, ldy = _matrix(y, "y", like)[:2]
        sp, lds = _opt_matrix(sum_out, "sum_out", like)
        _check(_lib.fa_layer_norm_forward(
            xp, ldx, rp, ldr, _CODES[x.dtype], rows, cols, wp, bp, pcode, eps, yp, ldy, sp, lds,
            _vector(mean, rows, "mean", dev, torch.float32), _vector(rstd, rows, "rstd", dev, torch.float32),
            _opt_checkpoint(ck_sum, rows, cols, "ck_sum", dev), _opt_checkpoint(ck_y, rows, cols, "ck_y", dev),
            _handle(dev)), "fa_layer_norm_forward")
    return y, mean, rstd, x if sum_out is None else sum_out


def fa_layer_norm_backward_workspace_bytes(rows: int, cols: int) -> int:
    return _bytes_of("fa_layer_norm_backward_workspace_bytes", rows, cols)


def fa_layer_norm_backward(dy, weight, mean, rstd, x=None, ck=None, residual_grad=None, dx=None, dweight=None, dbias=None,
                           ws=None, stream=None):
    """Gradient of fa_layer_norm_forward from its s (x) or the checkpoint of it (ck): (dx, dweight, dbias).

    residual_grad is added to dx: the gradient that reaches s past the norm.
    """
    dyp, lddy, rows, cols = _matrix(dy, "dy")
    dev = dy.device
    like = (rows, cols, dy.dtype, dev)
    if (x is None) == (ck is None):
        raise ValueError("exactly one of x and ck must be given")
    xp, ldx = _opt_matrix(x, "x", like)
    cp = _opt_checkpoint(ck, rows, cols, "ck", dev)
    rp, ldr = _opt_matrix(residual_grad, "residual_grad", like)
    wp, _, pcode = _params(weight, None, cols, ("weight", ""), dev)
    mp, sp = _vector(mean, rows, "mean", dev, torch.float32), _vector(rstd, rows, "rstd", dev, torch.float32)
    with _on(dev, stream):
        dx = torch.empty(dy.shape, dtype=dy.dtype, device=dev) if dx is None else dx
        dxp, lddx = _matrix(dx, "dx", like)[:2]
        (dweight, dbias), (dwp, dbp), gcode = _grads(dweight, dbias, ((cols,), (cols,)), ("dweight", "dbias"), dev)
        ws, wsp, wsb = _workspace(ws, fa_layer_norm_backward_workspace_bytes(rows, cols), dev)
        _check(_lib.fa_layer_norm_backward(
            dyp, lddy, xp, ldx, cp, _CODES[dy.dtype], rows, cols, wp, pcode, mp, sp, rp, ldr, dxp, lddx, dwp, dbp, gcode,
            wsp, wsb, _handle(dev)), "fa_layer_norm_backward")
    return dx, dweight, dbias


def fa_gelu_forward(x, bias=None, approximate="tanh", y=None, ck_x=None, ck_y=None, stream=None):
    """gelu(x + bias); ck_x / ck_y receive the checkpoints of x + bias and of the result."""
    xp, ldx, rows, cols = _matrix(x, "x")
    dev = x.device
    form = _approximate(approximate)
    bp, _, pcode = _params(bias, None, cols, ("bias", ""), dev)
    with _on(dev, stream):
        y = torch.empty(x.shape, dtype=x.dtype, device=dev) if y is None else y
        yp, ldy = _matrix(y, "y", (rows, cols, x.dtype, dev))[:2]
        _check(_lib.fa_gelu_forward(
            xp, ldx, _CODES[x.dtype], rows, cols, bp, pcode, form, yp, ldy, _opt_checkpoint(ck_x, rows, cols, "ck_x", dev),
            _opt_checkpoint(ck_y, rows, cols, "ck_y", dev), _handle(dev)), "fa_gelu_forward")
    return y


def fa_gelu_backward_workspace_bytes(rows: int, cols: int) -> int:
    return _bytes_of("fa_gelu_backward_workspace_bytes", rows, cols)


def fa_gelu_backward(dy, x=None, bias=None, ck=None, approximate="tanh", dx=None, dbias=None, ws=None, stream=None):
    """(dx, dbias) of fa_gelu_forward from its x and bias, or from ck_x, which holds their sum."""
    dyp, lddy, rows, cols = _matrix(dy, "dy")
    dev = dy.device
    like = (rows, cols, dy.dtype, dev)
    form = _approximate(approximate)
    if (x is None) == (ck is None):
        raise ValueError("exactly one of x and ck must be given")
    if ck is not None and bias is not None:
        raise ValueError("a checkpoint holds the input with its bias: bias must be None with ck")
    xp, ldx = _opt_matrix(x, "x", like)
    cp = _opt_checkpoint(ck, rows, cols, "ck", dev)
    bp, _, pcode = _params(bias, None, cols, ("bias", ""), dev)
    with _on(dev, stream):
        dx = torch.empty(dy.shape, dtype=dy.dtype, device=dev) if dx is None else dx
        dxp, lddx = _matrix(dx, "dx", like)[:2]
        (dbias, _), (dbp, _), gcode = _grads(dbias, False, ((cols,), ()), ("dbias", ""), dev)
        wsp, wsb = None, 0
        if dbias is not None:
            ws, wsp, wsb = _workspace(ws, fa_gelu_backward_workspace_bytes(rows, cols), dev)
        _check(_lib.fa_gelu_backward(
            dyp, lddy, xp, ldx, bp, pcode, cp, _CODES[dy.dtype], rows, cols, form, dxp, lddx, dbp, gcode, wsp, wsb,
            _handle(dev)), "fa_gelu_backward")
    return dx, dbias


def fa_linear_weight_grad_workspace_bytes(rows: int, outs: int, ins: int, dtype) -> int:
    return _bytes_of("fa_linear_weight_grad_workspace_bytes", rows, outs, ins, _CODES[dtype])


def fa_linear_weight_grad(dy, ck, ins, dweight=None, dbias=None, ws=None, stream=None):
    """(dweight, dbias) of a linear layer: dy^T X and the column sums of dy, X (rows x ins) as held by ck."""
    dyp, lddy, rows, outs = _matrix(dy, "dy")
    dev = dy.device
    cp = _buffer(ck, fa_checkpoint8_bytes(rows, ins), "ck", dev)
    if dweight is False:
        raise ValueError("dweight cannot be left out")
    with _on(dev, stream):
        (dweight, dbias), (dwp, dbp), gcode = _grads(dweight, dbias, ((outs, ins), (outs,)), ("dweight", "dbias"), dev)
        ws, wsp, wsb = _workspace(ws, fa_linear_weight_grad_workspace_bytes(rows, outs, ins, dy.dtype), dev)
        _check(_lib.fa_linear_weight_grad(dyp, lddy, _CODES[dy.dtype], rows, outs, cp, ins, dwp, dbp, gcode, wsp, wsb,
                                          _handle(dev)), "fa_linear_weight_grad")
    return dweight, dbias
