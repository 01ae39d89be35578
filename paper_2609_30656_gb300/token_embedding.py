"""Token lookup in one table, scaled, and the dense gradient of the table.

The Python binding of ``cb_token_forward`` / ``cb_token_backward`` (include/cb_tbe.h):

    x = token_forward(table, tokens, scale=math.sqrt(dim))        # [..., dim]
    dE = token_backward(grad_x, tokens, table.shape[0], scale=math.sqrt(dim))

Autograd records nothing of them: the second is the first's derivative, called by hand. Every
value is computed in fp32 and rounded once to the output's type. All work is
enqueued on the current stream of the tensors' device; nothing waits.
"""

from __future__ import annotations

import ctypes

import torch

from . import tbe

# The entry points of include/cb_tbe.h that this module binds.
EXPORTS = ("cb_token_forward", "cb_token_backward", "cb_token_backward_workspace_bytes")

_bound = None


def _library() -> ctypes.CDLL:
    global _bound
    if _bound is None:
        lib = tbe.load_library()
        p, i64, f32, c = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_int
        lib.cb_token_forward.argtypes = [p, c, i64, i64, i64, p, c, i64, i64, i64, i64, f32, p, c, i64, i64, p, p]
        lib.cb_token_backward.argtypes = [p, c, i64, i64, p, c, i64, i64, i64, i64, i64, i64, f32, i64, c, p, c, i64,
                                          p, i64, p, p]
        lib.cb_token_backward_workspace_bytes.argtypes = [i64, i64, i64]
        lib.cb_token_forward.restype = lib.cb_token_backward.restype = c
        lib.cb_token_backward_workspace_bytes.restype = i64
        _bound = lib
    return _bound


# A call here launches one kernel or a few, so on small batches the binding's own time is the
# call's: tensors' devices are compared by number, and contiguous tokens (one sequence to the
# library) are told apart first.
def _check_tokens(tokens: torch.Tensor, index: int) -> int:
    kind = tbe._IDX.get(tokens.dtype)
    if kind is None or tokens.get_device() != index:
        raise ValueError("tokens must be int32 or int64 on the device of the other tensors")
    return kind


def _check_error(error: torch.Tensor, index: int):
    if error.get_device() != index or error.dtype != torch.int32 or error.numel() != 1:
        raise ValueError("error must be an int32 tensor of one value on the device")


def _dtype(t: torch.Tensor, what: str) -> int:
    kind = tbe._DTYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"unsupported {what} dtype {t.dtype}")
    return kind


def _as_sequences(t: torch.Tensor, dims: int):
    """(tensor, sequences, length, sequence stride, place stride) of the leading `dims`
    dimensions; copies only what two strides cannot describe."""
    if dims > 2:
        t = t.flatten(0, dims - 2)  # a view wherever one can be made
    shape, stride = t.shape, t.stride()
    if dims == 0:
        return t, 1, 1, 0, 0
    if dims == 1:
        return t, 1, shape[0], 0, stride[0]
    return t, shape[0], shape[1], stride[0], stride[1]


def token_forward(table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, out: torch.Tensor | None = None,
                  out_dtype: torch.dtype | None = None, error: torch.Tensor | None = None) -> torch.Tensor:
    """out[..., :] = scale * table[tokens[...], :] (cb_token_forward).

    table: [rows, dim], fp32 / fp16 / bf16, rows contiguous, any row stride. tokens: int32 or
    int64 of any shape. out: [*tokens.shape, dim] of out_dtype (default: the table's type),
    rows contiguous. A token outside [0, rows) gives zeros and sets `error` (an int32 tensor of
    one value on the device) to CB_ERR_INDEX_OOB if it holds 0."""
    lib = _bound or _library()
    index = table.get_device()
    if index < 0 or table.dim() != 2:
        raise ValueError("table must be a 2-D CUDA tensor [rows, dim]")
    table_dtype = _dtype(table, "table")
    index_dtype = _check_tokens(tokens, index)
    if error is not None:
        _check_error(error, index)
    rows, dim = table.shape
    row_stride, step = table.stride()
    if dim > 1 and step != 1:
        raise ValueError("table rows must be contiguous")
    if rows <= 1:
        row_stride = dim
    elif row_stride < dim:
        raise ValueError("table rows must not overlap")
    fresh = out is None
    if fresh:
        out = torch.empty((*tokens.shape, dim), dtype=out_dtype or table.dtype, device=table.device)
    else:
        if out.get_device() != index or out.shape != (*tokens.shape, dim) or (dim > 1 and out.stride(-1) != 1):
            raise ValueError("out must be [*tokens.shape, dim] on the table's device, its rows contiguous")
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError(f"out must be {out_dtype}")
    kind = _dtype(out, "output")
    if tokens.is_contiguous() and (fresh or out.is_contiguous()):
        tok, sequences, length, tok0, tok1, out0, out1 = tokens, 1, tokens.numel(), 0, 1, 0, dim
    else:
        n_dims = tokens.dim()
        tok, sequences, length, tok0, tok1 = _as_sequences(tokens, n_dims)
        target, _, _, out0, out1 = _as_sequences(out, n_dims)
        if n_dims > 2 and target.data_ptr() != out.data_ptr():
            raise ValueError("out must be describable by two strides and contiguous rows")
    with tbe._OnDevice(index):
        status = lib.cb_token_forward(table.data_ptr(), table_dtype, rows, dim, row_stride, tok.data_ptr(), index_dtype,
                                      sequences, length, tok0, tok1, scale, out.data_ptr(), kind, out0, out1,
                                      None if error is None else error.data_ptr(), tbe._raw_stream(index))
    if status:
        tbe._check(status, "cb_token_forward")
    return out


def token_backward(grad_out: torch.Tensor, tokens: torch.Tensor, num_rows: int, scale: float = 1.0,
                   padding_idx: int | None = None, out: torch.Tensor | None = None,
                   out_dtype: torch.dtype | None = None, accumulate: bool = False,
                   error: torch.Tensor | None = None) -> torch.Tensor:
    """The gradient of token_forward with respect to the table, [num_rows, dim]:
    out[v] = scale * (sum of grad_out over the positions whose token is v) (cb_token_backward),
    fp32 unless out or out_dtype is of another type.

    With accumulate=True that is added to `out` in place and rows without a token are left
    alone; otherwise every row is written. Positions that hold padding_idx give nothing, nor
    do tokens outside [0, num_rows), which set `error` as in token_forward."""
    lib = _bound or _library()
    index = grad_out.get_device()
    shape = grad_out.shape
    if index < 0 or not shape or shape[:-1] != tokens.shape:
        raise ValueError("grad_out must be a CUDA tensor [*tokens.shape, dim]")
    go_dtype = _dtype(grad_out, "gradient")
    index_dtype = _check_tokens(tokens, index)
    if error is not None:
        _check_error(error, index)
    dim = shape[-1]
    if num_rows < 0:
        raise ValueError("num_rows must not be negative")
    if padding_idx is None:
        padding_idx = -1
    elif not 0 <= padding_idx < num_rows:
        raise ValueError("padding_idx must be a row of the table")
    row_stride = dim
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the gradient to add to")
        out = torch.empty(num_rows, dim, dtype=out_dtype or torch.float32, device=grad_out.device)
    else:
        if out.get_device() != index or out.shape != (num_rows, dim):
            raise ValueError("out must be [num_rows, dim] on the gradient's device")
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError(f"out must be {out_dtype}")
        if num_rows > 1:
            row_stride = out.stride(0)
        if (dim > 1 and out.stride(1) != 1) or row_stride < dim:
            raise ValueError("out's rows must be contiguous and must not overlap")
    kind = _dtype(out, "gradient")
    if tokens.is_contiguous() and grad_out.is_contiguous():
        tok, sequences, length, tok0, tok1, go, go0, go1 = tokens, 1, tokens.numel(), 0, 1, grad_out, 0, dim
    else:
        if dim > 1 and grad_out.stride(-1) != 1:
            grad_out = grad_out.contiguous()
        n_dims = tokens.dim()
        tok, sequences, length, tok0, tok1 = _as_sequences(tokens, n_dims)
        go, _, _, go0, go1 = _as_sequences(grad_out, n_dims)
    nbytes = lib.cb_token_backward_workspace_bytes(sequences * length, num_rows, dim)
    work = torch.empty(nbytes, dtype=torch.uint8, device=grad_out.device) if nbytes else None
    with tbe._OnDevice(index):
        status = lib.cb_token_backward(go.data_ptr(), go_dtype, go0, go1, tok.data_ptr(), index_dtype, sequences, length,
                                       tok0, tok1, num_rows, dim, scale, padding_idx, accumulate, out.data_ptr(), kind,
                                       row_stride, None if work is None else work.data_ptr(), nbytes,
                                       None if error is None else error.data_ptr(), tbe._raw_stream(index))
    if status:
        tbe._check(status, "cb_token_backward")
    return out
