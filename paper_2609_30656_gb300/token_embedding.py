"""Token lookup in one table, scaled, and the dense gradient of the table.

The Python binding of ``cb_token_forward`` / ``cb_token_backward`` (include/cb_tbe.h):

    x = token_forward(table, tokens, scale=math.sqrt(dim))        # [..., dim]
    dE = token_backward(grad_x, tokens, table.shape[0], scale=math.sqrt(dim))

Every value is computed in fp32 and rounded once to the output's type. All work is
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
        p, i32, i64, f32, c = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_int
        lib.cb_token_forward.argtypes = [p, c, i64, i32, i64, p, c, i32, i32, i64, i64, f32, p, c, i64, i64, p, p]
        lib.cb_token_backward.argtypes = [p, c, i64, i64, p, c, i32, i32, i64, i64, i64, i32, f32, i64, c, p, c, i64,
                                          p, i64, p, p]
        lib.cb_token_backward_workspace_bytes.argtypes = [i64, i64, i32]
        lib.cb_token_forward.restype = lib.cb_token_backward.restype = c
        lib.cb_token_backward_workspace_bytes.restype = i64
        _bound = lib
    return _bound


def _check_tokens(tokens: torch.Tensor, device: torch.device):
    if tokens.device != device or tokens.dtype not in tbe._IDX:
        raise ValueError("tokens must be int32 or int64 on the device of the other tensors")


def _check_error(error: torch.Tensor | None, device: torch.device):
    if error is not None and (error.device != device or error.dtype != torch.int32 or error.numel() != 1):
        raise ValueError("error must be an int32 tensor of one value on the device")


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


def _check_values(t: torch.Tensor, what: str):
    if t.dtype not in tbe._DTYPES:
        raise ValueError(f"unsupported {what} dtype {t.dtype}")


def token_forward(table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, out: torch.Tensor | None = None,
                  out_dtype: torch.dtype | None = None, error: torch.Tensor | None = None) -> torch.Tensor:
    """out[..., :] = scale * table[tokens[...], :] (cb_token_forward).

    table: [rows, dim], fp32 / fp16 / bf16, rows contiguous, any row stride. tokens: int32 or
    int64 of any shape. out: [*tokens.shape, dim] of out_dtype (default: the table's type),
    rows contiguous. A token outside [0, rows) gives zeros and sets `error` (an int32 tensor of
    one value on the device) to CB_ERR_INDEX_OOB if it holds 0."""
    lib = _library()
    if table.device.type != "cuda" or table.dim() != 2:
        raise ValueError("table must be a 2-D CUDA tensor [rows, dim]")
    _check_values(table, "table")
    _check_tokens(tokens, table.device)
    _check_error(error, table.device)
    rows, dim = table.shape
    if dim > 1 and table.stride(1) != 1:
        raise ValueError("table rows must be contiguous")
    if rows > 1 and table.stride(0) < dim:
        raise ValueError("table rows must not overlap")
    shape = (*tokens.shape, dim)
    if out is None:
        out = torch.empty(shape, dtype=out_dtype or table.dtype, device=table.device)
    else:
        if out.device != table.device or tuple(out.shape) != shape or (dim > 1 and out.stride(-1) != 1):
            raise ValueError("out must be [*tokens.shape, dim] on the table's device, its rows contiguous")
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError(f"out must be {out_dtype}")
    _check_values(out, "output")
    n_dims = tokens.dim()
    tok, sequences, length, tok0, tok1 = _as_sequences(tokens, n_dims)
    target, _, _, out0, out1 = _as_sequences(out, n_dims)
    if n_dims > 2 and target.data_ptr() != out.data_ptr():
        raise ValueError("out must be describable by two strides and contiguous rows")
    index = table.get_device()
    with tbe._OnDevice(index):
        tbe._check(lib.cb_token_forward(table.data_ptr(), tbe._DTYPES[table.dtype], rows, dim,
                                        table.stride(0) if rows > 1 else dim, tok.data_ptr(), tbe._IDX[tok.dtype],
                                        sequences, length, tok0, tok1, scale, out.data_ptr(), tbe._DTYPES[out.dtype],
                                        out0, out1, tbe._ptr(error), tbe._raw_stream(index)), "cb_token_forward")
    return out


def token_backward(grad_out: torch.Tensor, tokens: torch.Tensor, num_rows: int, scale: float = 1.0,
                   padding_idx: int | None = None, out: torch.Tensor | None = None,
                   out_dtype: torch.dtype = torch.float32, accumulate: bool = False,
                   error: torch.Tensor | None = None) -> torch.Tensor:
    """The gradient of token_forward with respect to the table, [num_rows, dim]:
    out[v] = scale * (sum of grad_out over the positions whose token is v) (cb_token_backward).

    With accumulate=True that is added to `out` in place and rows without a token are left
    alone; otherwise every row is written. Positions that hold padding_idx give nothing, nor
    do tokens outside [0, num_rows), which set `error` as in token_forward."""
    lib = _library()
    if grad_out.device.type != "cuda" or grad_out.dim() != tokens.dim() + 1 or grad_out.shape[:-1] != tokens.shape:
        raise ValueError("grad_out must be a CUDA tensor [*tokens.shape, dim]")
    _check_values(grad_out, "gradient")
    _check_tokens(tokens, grad_out.device)
    _check_error(error, grad_out.device)
    dim = grad_out.shape[-1]
    if num_rows < 0:
        raise ValueError("num_rows must not be negative")
    if padding_idx is not None and not 0 <= padding_idx < num_rows:
        raise ValueError("padding_idx must be a row of the table")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the gradient to add to")
        out = torch.empty(num_rows, dim, dtype=out_dtype, device=grad_out.device)
    elif (out.device != grad_out.device or tuple(out.shape) != (num_rows, dim) or (dim > 1 and out.stride(1) != 1)
          or (num_rows > 1 and out.stride(0) < dim)):
        raise ValueError("out must be [num_rows, dim] on the gradient's device, its rows contiguous")
    _check_values(out, "gradient")
    if dim > 1 and grad_out.stride(-1) != 1:
        grad_out = grad_out.contiguous()
    n_dims = tokens.dim()
    tok, sequences, length, tok0, tok1 = _as_sequences(tokens, n_dims)
    go, _, _, go0, go1 = _as_sequences(grad_out, n_dims)
    index = grad_out.get_device()
    nbytes = lib.cb_token_backward_workspace_bytes(sequences * length, num_rows, dim)
    work = torch.empty(nbytes, dtype=torch.uint8, device=grad_out.device) if nbytes else None
    with tbe._OnDevice(index):
        tbe._check(lib.cb_token_backward(go.data_ptr(), tbe._DTYPES[go.dtype], go0, go1, tok.data_ptr(),
                                         tbe._IDX[tok.dtype], sequences, length, tok0, tok1, num_rows, dim, scale,
                                         -1 if padding_idx is None else padding_idx, int(accumulate), out.data_ptr(),
                                         tbe._DTYPES[out.dtype], out.stride(0) if num_rows > 1 else dim,
                                         tbe._ptr(work), nbytes, tbe._ptr(error), tbe._raw_stream(index)),
                   "cb_token_backward")
    return out
