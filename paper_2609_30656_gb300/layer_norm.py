"""Layer normalisation of rows, and its backward pass with the gradients of weight and bias.

The Python binding of ``cb_layer_norm_forward`` / ``cb_layer_norm_backward`` (include/cb_tbe.h):

    y, mean, rstd = layer_norm(x, weight, bias, stats=True)                  # [..., dim]; fp32 [...]
    dx, dweight, dbias = layer_norm_backward(grad_y, x, mean, rstd, weight)

Autograd records nothing of them: the second is the first's derivative, called by hand. Every
value is computed in fp32 and rounded once to the output's type. All work is enqueued on the
current stream of the tensors' device; nothing waits.
"""

from __future__ import annotations

import ctypes

import torch

from . import tbe

# The entry points of include/cb_tbe.h that this module binds.
EXPORTS = ("cb_layer_norm_forward", "cb_layer_norm_backward", "cb_layer_norm_backward_workspace_bytes")

_bound = None


def _library() -> ctypes.CDLL:
    global _bound
    if _bound is None:
        lib = tbe.load_library()
        p, i64, f32, c = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_int
        lib.cb_layer_norm_forward.argtypes = [p, c, i64, i64, i64, p, c, p, c, f32, p, c, i64, p, p, p]
        lib.cb_layer_norm_backward.argtypes = [p, p, c, i64, i64, i64, i64, p, p, p, c, p, c, i64, p, p, p, i64, p]
        lib.cb_layer_norm_backward_workspace_bytes.argtypes = [i64, i64]
        lib.cb_layer_norm_forward.restype = lib.cb_layer_norm_backward.restype = c
        lib.cb_layer_norm_backward_workspace_bytes.restype = i64
        _bound = lib
    return _bound


def _dtype(t: torch.Tensor, what: str) -> int:
    kind = tbe._DTYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"unsupported {what} dtype {t.dtype}")
    return kind


def _as_rows(t: torch.Tensor):
    """(tensor, row stride) of [..., dim] as rows, or None if one stride does not describe them."""
    if t.is_contiguous():
        return t, t.shape[-1]
    shape, stride = t.shape, t.stride()
    if shape[-1] > 1 and stride[-1] != 1:
        return None
    step = rows = None
    for n, s in zip(reversed(shape[:-1]), reversed(stride[:-1])):
        if n == 1:
            continue
        if step is None:
            step, rows = s, n
        elif s != step * rows:
            return None
        else:
            rows *= n
    if step is None:
        step = shape[-1]
    return (t, step) if step >= shape[-1] else None


# One kernel or two are launched, so on small batches the binding's own time is the call's: contiguous
# tensors, the usual ones, are told apart first.
def _param(t: torch.Tensor | None, what: str, dim: int, index: int):
    if t is None:
        return None, 0
    kind = tbe._DTYPES.get(t.dtype)
    if t.get_device() != index or t.dim() != 1 or t.numel() != dim or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous, [dim], on the device of x")
    if kind is None:
        raise ValueError(f"unsupported {what} dtype {t.dtype}")
    return t.data_ptr(), kind


def _output(like: torch.Tensor, out: torch.Tensor | None, out_dtype: torch.dtype | None, index: int, what: str):
    """(tensor, row stride) of a result in the shape of `like`."""
    shape = like.shape
    if out is None:
        return torch.empty(shape, dtype=out_dtype or like.dtype, device=like.device), shape[-1]
    if out.get_device() != index or out.shape != shape:
        raise ValueError(f"{what} must have x's shape and device")
    if out_dtype is not None and out.dtype != out_dtype:
        raise TypeError(f"{what} must be {out_dtype}")
    rows = _as_rows(out)
    if rows is None:
        raise ValueError(f"{what} must have contiguous rows, equally far apart, that do not overlap")
    return rows


def layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, eps: float = 1e-5,
               out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None, stats: bool = False):
    """weight * (x - mean) * rstd + bias over the last dimension of x [..., dim] (cb_layer_norm_forward),
    in x's type unless out or out_dtype is of another.

    x: fp32 / fp16 / bf16; rows that are not contiguous or not equally far apart are copied. weight,
    bias: [dim], any of the three types, or None (1 and 0). out may be x. With stats=True the result is
    (out, mean, rstd), the latter two fp32 of shape [...], as the backward pass takes them."""
    lib = _bound or _library()
    index = x.get_device()
    if index < 0 or x.dim() < 1:
        raise ValueError("x must be a CUDA tensor [..., dim]")
    kind = _dtype(x, "x")
    shape = x.shape
    dim = shape[-1]
    w, w_kind = _param(weight, "weight", dim, index)
    b, b_kind = _param(bias, "bias", dim, index)
    fresh = out is None
    out, out_step = _output(x, out, out_dtype, index, "out")
    out_kind = _dtype(out, "output")
    if not fresh and out.data_ptr() == x.data_ptr() and x.numel() and (out.dtype != x.dtype or out.stride() != x.stride()):
        raise ValueError("out may be x, but not share its memory in another type or layout")
    step = dim
    if not x.is_contiguous():
        rows_of = _as_rows(x)
        x, step = rows_of if rows_of is not None else (x.contiguous(), dim)
    rows = x.numel() // dim if dim else 0
    mean = rstd = None
    if stats:
        device = x.device
        mean = torch.empty(shape[:-1], dtype=torch.float32, device=device)
        rstd = torch.empty(shape[:-1], dtype=torch.float32, device=device)
        if not dim:
            mean.zero_()
            rstd.fill_(float("inf") if eps == 0 else eps ** -0.5)
    with tbe._OnDevice(index):
        status = lib.cb_layer_norm_forward(x.data_ptr(), kind, rows, dim, step, w, w_kind, b, b_kind, eps, out.data_ptr(),
                                           out_kind, out_step, None if mean is None else mean.data_ptr(),
                                           None if rstd is None else rstd.data_ptr(), tbe._raw_stream(index))
    if status:
        tbe._check(status, "cb_layer_norm_forward")
    return (out, mean, rstd) if stats else out


def layer_norm_backward(grad_out: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                        weight: torch.Tensor | None = None, bias: bool = True, out: torch.Tensor | None = None,
                        out_dtype: torch.dtype | None = None):
    """The gradients (dx, dweight, dbias) of layer_norm, from the mean and rstd of its stats=True
    (cb_layer_norm_backward).

    grad_out has x's shape and type; dx too, unless out or out_dtype is of another (out may be grad_out or
    x). dweight and dbias are fp32 [dim]: dweight is None where there is no weight, dbias with bias=False."""
    lib = _bound or _library()
    index = x.get_device()
    if index < 0 or x.dim() < 1:
        raise ValueError("x must be a CUDA tensor [..., dim]")
    kind = _dtype(x, "x")
    if grad_out.get_device() != index or grad_out.shape != x.shape or grad_out.dtype != x.dtype:
        raise ValueError("grad_out must have x's shape, type and device")
    dim = x.shape[-1]
    for t, what in ((mean, "mean"), (rstd, "rstd")):
        if t.get_device() != index or t.dtype != torch.float32 or t.shape != x.shape[:-1]:
            raise ValueError(f"{what} must be fp32, x.shape[:-1], on the device of x")
    w, w_kind = _param(weight, "weight", dim, index)
    given = out is not None
    out, out_step = _output(x, out, out_dtype, index, "out")
    out_kind = _dtype(out, "gradient")
    for t in (x, grad_out) if given else ():
        if out.data_ptr() == t.data_ptr() and t.numel() and (out.dtype != t.dtype or out.stride() != t.stride()):
            raise ValueError("out may be grad_out or x, but not share its memory in another type or layout")
    go, go_step, step = grad_out, dim, dim
    if not x.is_contiguous():
        rows_of = _as_rows(x)
        x, step = rows_of if rows_of is not None else (x.contiguous(), dim)
    if not go.is_contiguous():
        rows_of = _as_rows(go)
        go, go_step = rows_of if rows_of is not None else (go.contiguous(), dim)
    mean, rstd = mean.contiguous(), rstd.contiguous()
    rows = x.numel() // dim if dim else 0
    dweight = torch.empty(dim, dtype=torch.float32, device=x.device) if weight is not None else None
    dbias = torch.empty(dim, dtype=torch.float32, device=x.device) if bias else None
    with tbe._OnDevice(index):
        nbytes, work = 0, None
        if (dweight is not None or dbias is not None) and rows:
            nbytes = lib.cb_layer_norm_backward_workspace_bytes(rows, dim)
            work = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
        status = lib.cb_layer_norm_backward(go.data_ptr(), x.data_ptr(), kind, rows, dim, go_step, step, mean.data_ptr(),
                                            rstd.data_ptr(), w, w_kind, out.data_ptr(), out_kind, out_step,
                                            None if dweight is None else dweight.data_ptr(),
                                            None if dbias is None else dbias.data_ptr(),
                                            None if work is None else work.data_ptr(), nbytes, tbe._raw_stream(index))
    if status:
        tbe._check(status, "cb_layer_norm_backward")
    return out, dweight, dbias
