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
_lib.fa_linear_weight_grad_workspace_bytes.argtypes = [_ll, _ll, _ll, _i, _i, ctypes.POINTER(_sz)]
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


def _matrix(t, name):
    """(pointer, row stride, rows, cols, type code, device) of the activation that sets a call's shape."""
    code = _code(t, name)
    shape = t.shape
    if not shape or shape[-1] < 1:
        raise ValueError(f"{name} must have a last dimension of at least one element")
    cols = shape[-1]
    ld = cols if t.is_contiguous() else _row_stride(t, name)
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    return t.data_ptr(), ld, t.numel() // cols, cols, code, t.device


def _where(t, name, device):
    return ValueError(f"{name} must be a CUDA tensor" if not t.is_cuda else f"{name} is on {t.device}, the call runs on {device}")


def _like(t, name, rows, cols, dtype, device):
    """(pointer, row stride) of another activation of the same call."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    shape = t.shape
    if t.dtype is not dtype or not shape or shape[-1] != cols or t.numel() != rows * cols:
        raise ValueError(f"{name} must have {rows} rows of {cols} elements of {dtype}, got {tuple(shape)} of {t.dtype}")
    ld = cols if t.is_contiguous() else _row_stride(t, name)
    if t.get_device() != device.index:
        raise _where(t, name, device)
    return t.data_ptr(), ld


def _vector(t, numel, name, device, dtype=None):
    """Pointer of a contiguous tensor of exactly `numel` elements, of `dtype` or of either float type."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if dtype is None:
        if t.dtype not in _CODES:
            raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    elif t.dtype is not dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() != numel:
        raise ValueError(f"{name} must have {numel} elements, got {t.numel()}")
    if t.get_device() != device.index:
        raise _where(t, name, device)
    return t.data_ptr()


def _param(t, numel, name, device):
    """(pointer, type code) of an optional parameter vector."""
    return (None, FA_F32) if t is None else (_vector(t, numel, name, device), _CODES[t.dtype])


def _buffer(t, nbytes, name, device):
    """Pointer of a byte buffer (checkpoint, workspace) of at least nbytes."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.nbytes < nbytes:
        raise ValueError(f"{name} must have at least {nbytes} bytes, got {t.nbytes}")
    if not t.is_cuda or t.get_device() != device.index:
        raise _where(t, name, device)
    return t.data_ptr()


def _opt_checkpoint(t, rows, cols, name, device):
    return None if t is None else _buffer(t, _bytes_of("fa_checkpoint8_bytes", rows, cols), name, device)


def _grad(t, shape, numel, name, device, partner=None):
    """(tensor or None, pointer) of a parameter gradient (see the module's docstring for None and False)."""
    if t is False:
        return None, None
    if t is None:
        like = partner if isinstance(partner, torch.Tensor) else None
        t = torch.empty(shape, dtype=torch.float32 if like is None else like.dtype, device=device)
        return t, t.data_ptr()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor, None or False")
    return t, _vector(t, numel, name, device)


def _grad_code(first, second, names):
    """Common type code of two gradients, either of which may be None."""
    one = first if first is not None else second
    if one is None:
        return FA_F32
    if first is not None and second is not None and first.dtype != second.dtype:
        raise ValueError(f"{names} must have the same dtype")
    return _CODES[one.dtype]


def _on(device, stream):
    """Context in which a call allocates and launches."""
    if stream is None:
        return _HERE if torch.cuda.current_device() == device.index else torch.cuda.device(device)
    if stream.device != device:
        raise ValueError(f"stream belongs to {stream.device}, the tensors are on {device}")
    return torch.cuda.stream(stream)


# handle of the current stream (torch.cuda.current_stream(device).cuda_stream is a fifth of a small call's time)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _fresh(like):
    """A dense tensor of the shape and type of `like`."""
    return torch.empty_like(like, memory_format=torch.contiguous_format)


def _workspace(ws, nbytes, device):
    if ws is None:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        return ws, ws.data_ptr(), nbytes
    return ws, _buffer(ws, nbytes, "ws", device), ws.nbytes


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
    xp, ldx, rows, cols, code, dev = _matrix(x, "x")
    with _on(dev, stream):
        nbytes = fa_checkpoint8_bytes(rows, cols)
        if ck is None:
            ck = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        _check(_lib.fa_checkpoint8_store(xp, ldx, code, rows, cols, _buffer(ck, nbytes, "ck", dev), _raw_stream(dev.index)),
               "fa_checkpoint8_store")
    return ck


def fa_checkpoint8_load(ck, rows, cols, out=None, dtype=torch.bfloat16, stream=None):
    """The rows x cols activations that ck holds, as `out` or a new tensor of `dtype`."""
    if not isinstance(ck, torch.Tensor):
        raise TypeError("ck must be a torch tensor")
    dev = ck.device
    cp = _buffer(ck, fa_checkpoint8_bytes(rows, cols), "ck", dev)
    with _on(dev, stream):
        if out is None:
            out = torch.empty((rows, cols), dtype=dtype, device=dev)
        code = _code(out, "out")
        op, ldo = _like(out, "out", rows, cols, out.dtype, dev)
        _check(_lib.fa_checkpoint8_load(cp, code, rows, cols, op, ldo, _raw_stream(dev.index)), "fa_checkpoint8_load")
    return out


def fa_layer_norm_forward(x, weight=None, bias=None, eps=1e-5, residual=None, y=None, sum_out=None, mean=None, rstd=None,
                          ck_sum=None, ck_y=None, stream=None):
    """Layer norm of s = x + residual; returns (y, mean, rstd, s).

    Without a residual s is x itself (sum_out None).  ck_sum / ck_y: buffers of new_checkpoint8() that
    receive the checkpoints of s and of y.
    """
    xp, ldx, rows, cols, code, dev = _matrix(x, "x")
    dtype = x.dtype
    rp, ldr = (None, 0) if residual is None else _like(residual, "residual", rows, cols, dtype, dev)
    wp, pcode = _param(weight, cols, "weight", dev)
    bp, bcode = _param(bias, cols, "bias", dev)
    if wp is None:
        pcode = bcode
    elif bp is not None and bcode != pcode:
        raise ValueError("weight and bias must have the same dtype")
    with _on(dev, stream):
        if y is None:
            y = _fresh(x)
            yp, ldy = y.data_ptr(), cols
        else:
            yp, ldy = _like(y, "y", rows, cols, dtype, dev)
        sp, lds = (None, 0) if sum_out is None else _like(sum_out, "sum_out", rows, cols, dtype, dev)
        if sum_out is None and residual is not None:
            sum_out = _fresh(x)
            sp, lds = sum_out.data_ptr(), cols
        if mean is None:
            mean = torch.empty(rows, dtype=torch.float32, device=dev)
        else:
            _vector(mean, rows, "mean", dev, torch.float32)
        if rstd is None:
            rstd = torch.empty(rows, dtype=torch.float32, device=dev)
        else:
            _vector(rstd, rows, "rstd", dev, torch.float32)
        _check(_lib.fa_layer_norm_forward(
            xp, ldx, rp, ldr, code, rows, cols, wp, bp, pcode, eps, yp, ldy, sp, lds, mean.data_ptr(), rstd.data_ptr(),
            _opt_checkpoint(ck_sum, rows, cols, "ck_sum", dev), _opt_checkpoint(ck_y, rows, cols, "ck_y", dev),
            _raw_stream(dev.index)), "fa_layer_norm_forward")
    return y, mean, rstd, x if sum_out is None else sum_out


def fa_layer_norm_backward_workspace_bytes(rows: int, cols: int) -> int:
    return _bytes_of("fa_layer_norm_backward_workspace_bytes", rows, cols)


def fa_layer_norm_backward(dy, weight, mean, rstd, x=None, ck=None, residual_grad=None, dx=None, dweight=None, dbias=None,
                           ws=None, stream=None):
    """Gradient of fa_layer_norm_forward from its s (x) or the checkpoint of it (ck): (dx, dweight, dbias).

    residual_grad is added to dx: the gradient that reaches s past the norm.
    """
    dyp, lddy, rows, cols, code, dev = _matrix(dy, "dy")
    dtype = dy.dtype
    if (x is None) == (ck is None):
        raise ValueError("exactly one of x and ck must be given")
    xp, ldx = (None, 0) if x is None else _like(x, "x", rows, cols, dtype, dev)
    cp = _opt_checkpoint(ck, rows, cols, "ck", dev)
    rp, ldr = (None, 0) if residual_grad is None else _like(residual_grad, "residual_grad", rows, cols, dtype, dev)
    wp, pcode = _param(weight, cols, "weight", dev)
    mp, sp = _vector(mean, rows, "mean", dev, torch.float32), _vector(rstd, rows, "rstd", dev, torch.float32)
    with _on(dev, stream):
        if dx is None:
            dx = _fresh(dy)
            dxp, lddx = dx.data_ptr(), cols
        else:
            dxp, lddx = _like(dx, "dx", rows, cols, dtype, dev)
        given = dbias
        dbias, dbp = _grad(dbias, (cols,), cols, "dbias", dev, dweight)
        dweight, dwp = _grad(dweight, (cols,), cols, "dweight", dev, given)
        ws, wsp, wsb = _workspace(ws, fa_layer_norm_backward_workspace_bytes(rows, cols), dev)
        _check(_lib.fa_layer_norm_backward(
            dyp, lddy, xp, ldx, cp, code, rows, cols, wp, pcode, mp, sp, rp, ldr, dxp, lddx, dwp, dbp,
            _grad_code(dweight, dbias, "dweight and dbias"), wsp, wsb, _raw_stream(dev.index)), "fa_layer_norm_backward")
    return dx, dweight, dbias


def fa_gelu_forward(x, bias=None, approximate="tanh", y=None, ck_x=None, ck_y=None, stream=None):
    """gelu(x + bias); ck_x / ck_y receive the checkpoints of x + bias and of the result."""
    xp, ldx, rows, cols, code, dev = _matrix(x, "x")
    form = _approximate(approximate)
    bp, pcode = _param(bias, cols, "bias", dev)
    with _on(dev, stream):
        if y is None:
            y = _fresh(x)
            yp, ldy = y.data_ptr(), cols
        else:
            yp, ldy = _like(y, "y", rows, cols, x.dtype, dev)
        _check(_lib.fa_gelu_forward(
            xp, ldx, code, rows, cols, bp, pcode, form, yp, ldy, _opt_checkpoint(ck_x, rows, cols, "ck_x", dev),
            _opt_checkpoint(ck_y, rows, cols, "ck_y", dev), _raw_stream(dev.index)), "fa_gelu_forward")
    return y


def fa_gelu_backward_workspace_bytes(rows: int, cols: int) -> int:
    return _bytes_of("fa_gelu_backward_workspace_bytes", rows, cols)


def fa_gelu_backward(dy, x=None, bias=None, ck=None, approximate="tanh", dx=None, dbias=None, ws=None, stream=None):
    """(dx, dbias) of fa_gelu_forward from its x and bias, or from ck_x, which holds their sum."""
    dyp, lddy, rows, cols, code, dev = _matrix(dy, "dy")
    dtype = dy.dtype
    form = _approximate(approximate)
    if (x is None) == (ck is None):
        raise ValueError("exactly one of x and ck must be given")
    if ck is not None and bias is not None:
        raise ValueError("a checkpoint holds the input with its bias: bias must be None with ck")
    xp, ldx = (None, 0) if x is None else _like(x, "x", rows, cols, dtype, dev)
    cp = _opt_checkpoint(ck, rows, cols, "ck", dev)
    bp, pcode = _param(bias, cols, "bias", dev)
    with _on(dev, stream):
        if dx is None:
            dx = _fresh(dy)
            dxp, lddx = dx.data_ptr(), cols
        else:
            dxp, lddx = _like(dx, "dx", rows, cols, dtype, dev)
        dbias, dbp = _grad(dbias, (cols,), cols, "dbias", dev)
        wsp, wsb = None, 0
        if dbias is not None:
            ws, wsp, wsb = _workspace(ws, fa_gelu_backward_workspace_bytes(rows, cols), dev)
        _check(_lib.fa_gelu_backward(
            dyp, lddy, xp, ldx, bp, pcode, cp, code, rows, cols, form, dxp, lddx, dbp, _grad_code(dbias, None, "dbias"),
            wsp, wsb, _raw_stream(dev.index)), "fa_gelu_backward")
    return dx, dbias


def fa_linear_weight_grad_workspace_bytes(rows: int, outs: int, ins: int, dtype, aligned: bool = False) -> int:
    """aligned: address and row stride of dy are multiples of 16 bytes, and the row stride is at least outs."""
    return _bytes_of("fa_linear_weight_grad_workspace_bytes", rows, outs, ins, _CODES[dtype], 1 if aligned else 0)


def fa_linear_weight_grad(dy, ck, ins, dweight=None, dbias=None, ws=None, stream=None):
    """(dweight, dbias) of a linear layer: dy^T X and the column sums of dy, X (rows x ins) as held by ck."""
    dyp, lddy, rows, outs, code, dev = _matrix(dy, "dy")
    cp = _buffer(ck, fa_checkpoint8_bytes(rows, ins), "ck", dev)
    if dweight is False:
        raise ValueError("dweight cannot be left out")
    with _on(dev, stream):
        given = dbias
        dbias, dbp = _grad(dbias, (outs,), outs, "dbias", dev, dweight)
        dweight, dwp = _grad(dweight, (outs, ins), outs * ins, "dweight", dev, given)
        aligned = 0 if dyp % 16 or lddy * dy.element_size() % 16 or lddy < outs else 1
        nbytes = _bytes_of("fa_linear_weight_grad_workspace_bytes", rows, outs, ins, code, aligned)
        ws, wsp, wsb = _workspace(ws, nbytes, dev)
        _check(_lib.fa_linear_weight_grad(dyp, lddy, code, rows, outs, cp, ins, dwp, dbp,
                                          _grad_code(dweight, dbias, "dweight and dbias"), wsp, wsb,
                                          _raw_stream(dev.index)), "fa_linear_weight_grad")
    return dweight, dbias
