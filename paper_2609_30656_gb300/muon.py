"""Orthogonalised matrix updates: Newton-Schulz products, and the optimizer step around them.

The Python binding of ``cb_muon_orthogonalise`` / ``cb_muon_step`` (include/cb_tbe.h). As the
library's other calls these compute and write in place; autograd records nothing of them.

    o = newton_schulz(g)                                  # about U V^T of g = U S V^T
    muon_step(weight, grad, momentum, lr=3e-4, weight_decay=0.1)

Matrices are 2-D, or 3-D for a stack of equal shapes. All work is enqueued on the current
stream of the tensors' device; nothing waits. The workspace (about 8 bytes per value of the
update and 4 per value of its square Gram matrix) comes from torch's allocator.
"""

from __future__ import annotations

import ctypes
import math

import torch

from . import tbe

# The entry points of include/cb_tbe.h that this module binds.
EXPORTS = ("cb_muon_orthogonalise", "cb_muon_step", "cb_muon_workspace_bytes")

COEFFICIENTS = (3.4445, -4.7750, 2.0315)  # every singular value in (0, 1] into about [0.7, 1.2] in five steps

_bound = None
_coefficient_arrays: dict = {}


def _library() -> ctypes.CDLL:
    global _bound
    if _bound is None:
        lib = tbe.load_library()
        p, i32, i64, f32, c = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_int
        lib.cb_muon_orthogonalise.argtypes = [p, c, i64, i64, i64, i64, i64, f32, p, i32, p, c, i64, i64, p, i64, p, p]
        lib.cb_muon_step.argtypes = [p, c, i64, i64, p, c, i64, i64, p, i64, i64, i64, i64, i64, f32, f32, f32, c,
                                     f32, p, i32, f32, p, i64, p, p]
        lib.cb_muon_workspace_bytes.argtypes = [i64, i64, i64]
        lib.cb_muon_orthogonalise.restype = lib.cb_muon_step.restype = c
        lib.cb_muon_workspace_bytes.restype = i64
        _bound = lib
    return _bound


def _coefficients(coefficients, steps: int):
    """A C array of 3 * steps values: one triple for all steps, or one for each."""
    key = (coefficients, steps) if type(coefficients) is tuple else None
    try:
        array = _coefficient_arrays.get(key)
    except TypeError:  # a tuple of lists
        key = array = None
    if array is not None:
        return array
    if steps < 1:
        raise ValueError("at least one step is needed")
    rows = tuple(coefficients)
    if len(rows) == 3 and not any(hasattr(x, "__len__") for x in rows):
        rows = (rows,) * steps
    if len(rows) != steps or any(not hasattr(r, "__len__") or len(r) != 3 for r in rows):
        raise ValueError("coefficients must be one triple, or one triple for each step")
    array = (ctypes.c_float * (3 * steps))(*[float(x) for r in rows for x in r])
    # Kept only where nothing in it can change.
    if key is not None and all(type(r) is tuple and all(type(x) in (float, int) for x in r) for r in rows):
        if len(_coefficient_arrays) >= 64:
            _coefficient_arrays.clear()
        _coefficient_arrays[key] = array
    return array


def _check_matrix(t: torch.Tensor, what: str) -> int:
    if t.get_device() < 0 or t.dim() not in (2, 3):
        raise ValueError(f"{what} must be a 2-D or 3-D CUDA tensor")
    kind = tbe._DTYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"unsupported {what} dtype {t.dtype}")
    return kind


def _check_error(error: torch.Tensor, index: int):
    if error.get_device() != index or error.dtype != torch.int32 or error.numel() != 1:
        raise ValueError("error must be an int32 tensor of one value on the device")


def _rows_apart(batch: int, batch_stride: int, rows: int, row_stride: int, cols: int) -> bool:
    """No value is in two rows: matrices one after the other, their rows in turn, or else no two rows too near."""
    if batch_stride < cols:
        return False
    if batch_stride >= (rows - 1) * row_stride + cols or row_stride >= (batch - 1) * batch_stride + cols:
        return True
    (n, step), (m, other) = sorted(((batch, batch_stride), (rows, row_stride)))
    for k in range(1, n):
        below, rest = divmod(k * step, other)
        if (below < m and rest < cols) or (below + 1 < m and other - rest < cols):
            return False
    return True


def _layout(t: torch.Tensor):
    """(batch stride, row stride, rows contiguous, no two values in one place) in values; a
    dimension of one has the stride of a whole one."""
    shape = t.shape
    rows, cols = shape[-2:]
    if t.is_contiguous():
        return rows * cols, cols, True, True
    stride = t.stride()
    row = stride[-2] if rows > 1 else cols
    many = t.dim() == 3 and shape[0] > 1
    batch = stride[0] if many else rows * row
    in_rows = (cols <= 1 or stride[-1] == 1) and row >= cols
    return batch, row, in_rows, in_rows and (not many or _rows_apart(shape[0], batch, rows, row, cols))


def newton_schulz(g: torch.Tensor, out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                  steps: int = 5, coefficients=COEFFICIENTS, eps: float = 1e-7,
                  error: torch.Tensor | None = None) -> torch.Tensor:
    """The approximate orthogonal factor of g, or of each matrix of a stack
    (cb_muon_orthogonalise), bf16 unless out or out_dtype is of another type.

    X = g / (||g||_F + eps), then `steps` times X <- a X + (b A + c A A) X with A = X X^T.
    The products are in fp16 with fp32 sums, 2e-4 to 2.8e-3 off the exact result in the 2-norm (most or all
    singular values alike: the most; a constant matrix 1.3e-2), which is why the default output type is bf16; a wider
    one is not more exact than that. out may be g. A g whose columns are
    contiguous (a transposed view) is taken as it lies."""
    lib = _bound or _library()
    kind = _check_matrix(g, "g")
    index = g.get_device()
    if error is not None:
        _check_error(error, index)
    layout = _layout(g)
    if out is None:
        out_dtype = out_dtype or torch.bfloat16
        if not layout[2] and _layout(g.mT)[2]:
            out = torch.empty(g.mT.shape, dtype=out_dtype, device=g.device).mT
        else:
            out = torch.empty(g.shape, dtype=out_dtype, device=g.device)
    elif out_dtype is not None and out.dtype != out_dtype:
        raise TypeError(f"out must be {out_dtype}")
    out_kind = _check_matrix(out, "out")
    out_layout = _layout(out)
    if out.get_device() != index or out.shape != g.shape or not (out_layout[3] or _layout(out.mT)[3]):
        raise ValueError("out must have g's shape and device, its rows or columns contiguous, its matrices apart")
    if not out_layout[3]:  # the transpose's factor is the factor's transpose
        newton_schulz(g.mT, out.mT, out.dtype, steps, coefficients, eps, error)
        return out
    if not layout[2]:
        g = g.contiguous()
        layout = _layout(g)
    shape = g.shape
    rows, cols = shape[-2:]
    batch = shape[0] if len(shape) == 3 else 1
    table = _coefficients(coefficients, steps)
    if g.numel() == 0:
        return out
    nbytes = lib.cb_muon_workspace_bytes(batch, rows, cols)
    work = torch.empty(nbytes, dtype=torch.uint8, device=g.device)
    with tbe._OnDevice(index):
        status = lib.cb_muon_orthogonalise(g.data_ptr(), kind, batch, rows, cols, layout[0], layout[1], eps, table, steps,
                                           out.data_ptr(), out_kind, out_layout[0], out_layout[1], work.data_ptr(), nbytes,
                                           None if error is None else error.data_ptr(), tbe._raw_stream(index))
    if status:
        tbe._check(status, "cb_muon_orthogonalise")
    return out


def update_scale(rows: int, cols: int, adjust: str | None) -> float:
    """What an orthogonalised update of shape [rows, cols] is multiplied with besides lr:
    "rms": 0.2 sqrt(max(rows, cols)), values of the size of an Adam step's; "spectral":
    sqrt(max(1, rows / cols)), the same change of the layer's outputs for every shape; None: 1."""
    if adjust == "rms":
        return 0.2 * math.sqrt(max(rows, cols))
    if adjust == "spectral":
        return math.sqrt(max(1.0, rows / cols))
    if adjust is None:
        return 1.0
    raise ValueError(f"unknown adjustment {adjust!r}")


def muon_step(weight: torch.Tensor, grad: torch.Tensor, momentum: torch.Tensor, lr: float, beta: float = 0.95,
              nesterov: bool = True, weight_decay: float = 0.0, adjust: str | None = "rms", steps: int = 5,
              coefficients=COEFFICIENTS, eps: float = 1e-7, error: torch.Tensor | None = None) -> None:
    """One optimizer step of a weight matrix, or of a stack of them, in place (cb_muon_step):

        momentum <- beta momentum + grad;  u = grad + beta momentum (nesterov) or momentum
        weight <- (1 - lr weight_decay) weight - lr update_scale(adjust) newton_schulz(u)

    weight and grad: fp32 / fp16 / bf16; momentum: fp32 (a running sum keeps its 32 bits).
    The three have one shape; weight and momentum have contiguous rows (a grad that has not is copied)."""
    lib = _bound or _library()
    index = weight.get_device()
    kinds = [_check_matrix(t, what) for t, what in ((weight, "weight"), (grad, "grad"), (momentum, "momentum"))]
    shape = weight.shape
    for t in (grad, momentum):
        if t.get_device() != index or t.shape != shape:
            raise ValueError("weight, grad and momentum must have one shape and device")
    if error is not None:
        _check_error(error, index)
    if momentum.dtype != torch.float32:
        raise ValueError("momentum must be fp32")
    w, m, g = _layout(weight), _layout(momentum), _layout(grad)
    if not w[3] or not m[3]:
        raise ValueError("weight and momentum must have contiguous rows and matrices that do not overlap")
    if not g[2]:
        grad = grad.contiguous()
        g = _layout(grad)
    rows, cols = shape[-2:]
    batch = shape[0] if len(shape) == 3 else 1
    table = _coefficients(coefficients, steps)
    scale = update_scale(rows, cols, adjust) if cols else 1.0
    if weight.numel() == 0:
        return
    nbytes = lib.cb_muon_workspace_bytes(batch, rows, cols)
    work = torch.empty(nbytes, dtype=torch.uint8, device=weight.device)
    with tbe._OnDevice(index):
        status = lib.cb_muon_step(weight.data_ptr(), kinds[0], w[0], w[1], grad.data_ptr(), kinds[1], g[0], g[1],
                                  momentum.data_ptr(), m[0], m[1], batch, rows, cols, lr, weight_decay, beta, nesterov,
                                  eps, table, steps, scale, work.data_ptr(), nbytes,
                                  None if error is None else error.data_ptr(), tbe._raw_stream(index))
    if status:
        tbe._check(status, "cb_muon_step")
