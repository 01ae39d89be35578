"""The norm over all gradients of a model, and the gradients clipped to it.

The Python binding of ``cb_grad_norm`` / ``cb_grad_clip`` (include/cb_tbe.h). As the library's other
calls these compute and write in place; nothing waits, and the norm stays on the device:

    norm = clip_grad_norm([dE, dW1, dW2, sparse], max_norm=1.0)       # fp32 tensor of one value
    norm = grad_norm(grads)

A gradient is a tensor, fp32 / fp16 / bf16, of any shape (dense, or rows equally far apart); a
``tbe.SparseGrad``, whose values count as far as its num_floats says; or a pair (fp32 values, int64 tensor of how
many of them count) for the same thing held otherwise.
"""

from __future__ import annotations

import ctypes
import struct

import torch

from . import tbe

# The entry points of include/cb_tbe.h that this module binds.
EXPORTS = ("cb_grad_norm", "cb_grad_clip", "cb_grad_norm_workspace_bytes")


class CbGradTensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("count", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("row_stride", ctypes.c_int64), ("out_row_stride", ctypes.c_int64),
                ("dtype", ctypes.c_int), ("out_dtype", ctypes.c_int)]


_bound = None


def _library() -> ctypes.CDLL:
    global _bound
    if _bound is None:
        lib = tbe.load_library()
        p, i64, f32, c = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_int
        lib.cb_grad_norm.argtypes = [p, i64, p, p, i64, p]
        lib.cb_grad_clip.argtypes = [p, i64, f32, f32, p, p, i64, p]
        lib.cb_grad_norm_workspace_bytes.argtypes = [i64]
        lib.cb_grad_norm.restype = lib.cb_grad_clip.restype = c
        lib.cb_grad_norm_workspace_bytes.restype = i64
        _bound = lib
    return _bound


def _as_rows(t: torch.Tensor, to: torch.Tensor):
    """(rows, cols, row stride of t, of to) of two tensors of one shape whose values lie alike, densely in
    some order of the dimensions or in rows equally far apart; None for any others."""
    n = t.numel()
    if n <= 1 or (t.is_contiguous() and (to is t or to.is_contiguous())):
        return 1, n, n, n
    dims = sorted((s, o, size) for size, s, o in zip(t.shape, t.stride(), to.stride()) if size > 1)
    cols = k = 1
    for k, (s, o, size) in enumerate(dims):
        if s != cols or o != cols:
            break
        cols *= size
    else:
        return 1, n, n, n
    step, out_step, rows = dims[k][0], dims[k][1], 1
    for s, o, size in dims[k:]:
        if s != step * rows or o != out_step * rows:
            return None
        rows *= size
    return (rows, cols, step, out_step) if step >= cols and out_step >= cols else None


def _values(g, what: str):
    """(tensor, count or None) of a gradient in one of its forms."""
    if isinstance(g, torch.Tensor):
        return g, None
    if isinstance(g, tbe.SparseGrad):
        if g.grads is None:
            raise ValueError("a size-only gradient holds no values")
        g = (g.grads, g.num_floats_dev)
    if not isinstance(g, (tuple, list)) or len(g) != 2 or not all(isinstance(t, torch.Tensor) for t in g):
        raise TypeError(f"{what} must be tensors, SparseGrads or pairs (values, count)")
    values, count = g
    if values.dtype != torch.float32 or not values.is_contiguous():
        raise ValueError("values that are counted must be fp32 and contiguous")
    if count.dtype != torch.int64 or count.numel() != 1 or count.get_device() != values.get_device():
        raise ValueError("a count must be an int64 tensor of one value on the device of its values")
    return values, count


def _listed(grads):
    return [grads] if isinstance(grads, (torch.Tensor, tbe.SparseGrad)) else list(grads)


# A small model has dozens of tensors, so their checks are most of a call's time: a contiguous one takes the short
# way, and the table is packed at once (with a ctypes structure filled field by field 20 tensors took 20 us more).
def _table(grads, out):
    """(the C table as bytes, its length, the device, the tensors in it) of the gradients and where they are written."""
    grads = _listed(grads)
    outs = grads if out is None else _listed(out)
    if len(outs) != len(grads):
        raise ValueError("out must hold a tensor for each gradient")
    if not grads:
        raise ValueError("at least one gradient is needed")
    words, kept = [], []
    index = None
    for g, o in zip(grads, outs):
        count = to_count = None
        t, to = g, o
        if type(t) is not torch.Tensor:
            t, count = _values(g, "gradients")
        if o is g:
            to = t
        elif type(to) is not torch.Tensor:
            to, to_count = _values(o, "outputs")
        device = t.get_device()
        if device != index:
            if device < 0 or index is not None:
                raise ValueError("gradients must be on one CUDA device")
            index = device
        kind = to_kind = tbe._DTYPES.get(t.dtype)
        if kind is None:
            raise ValueError(f"unsupported gradient dtype {t.dtype}")
        if o is not g:
            if to.get_device() != index or to.shape != t.shape or (count is None) != (to_count is None):
                raise ValueError("an output must have its gradient's form, shape and device")
            if count is not None and to_count.data_ptr() != count.data_ptr():
                raise ValueError("an output's count must be its gradient's")
            to_kind = tbe._DTYPES.get(to.dtype)
            if to_kind is None:
                raise ValueError(f"unsupported output dtype {to.dtype}")
        if t.is_contiguous() and (to is t or to.is_contiguous()):
            n = t.numel()
            rows = (1, n, n, n)
        else:
            rows = _as_rows(t, to)
            if rows is None:
                raise ValueError("a gradient's values must be dense, or in rows equally far apart that do not overlap, and an "
                                 "output's lie alike")
        ptr = t.data_ptr()
        words += (ptr, ptr if to is t else to.data_ptr(), 0 if count is None else count.data_ptr(), *rows, kind | to_kind << 32)
        kept.append((t, to, count))
    return struct.pack(f"{len(words)}q", *words), len(grads), index, kept


def _scratch(lib, n: int, index: int):
    """(norm, workspace, its bytes); the norm is alone in its memory."""
    device = torch.device("cuda", index)
    nbytes = lib.cb_grad_norm_workspace_bytes(n)
    return torch.empty((), dtype=torch.float32, device=device), torch.empty(nbytes, dtype=torch.uint8, device=device), nbytes


def grad_norm(grads) -> torch.Tensor:
    """sqrt(sum of x^2) over all values of all gradients, fp32, on their device (cb_grad_norm)."""
    lib = _bound or _library()
    table, n, index, _ = _table(grads, None)
    with tbe._OnDevice(index):
        norm, work, nbytes = _scratch(lib, n, index)
        status = lib.cb_grad_norm(table, n, norm.data_ptr(), work.data_ptr(), nbytes, tbe._raw_stream(index))
    if status:
        tbe._check(status, "cb_grad_norm")
    return norm


def clip_grad_norm(grads, max_norm: float, eps: float = 1e-6, out=None) -> torch.Tensor:
    """Every gradient times min(1, max_norm / (norm + eps)), in place, and the norm before that
    (cb_grad_clip). With `out`, one tensor (or SparseGrad, or pair) for each gradient, of any of
    the types, the products go there and the gradients stay as they are.

    A tensor may be in the list once. A norm that is not finite makes gradients of NaNs and zeros, which a
    caller who skips such steps does not use."""
    lib = _bound or _library()
    table, n, index, _ = _table(grads, out)
    with tbe._OnDevice(index):
        norm, work, nbytes = _scratch(lib, n, index)
        status = lib.cb_grad_clip(table, n, max_norm, eps, norm.data_ptr(), work.data_ptr(), nbytes, tbe._raw_stream(index))
    if status:
        tbe._check(status, "cb_grad_clip")
    return norm
