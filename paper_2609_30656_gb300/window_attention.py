"""Causal attention within the sessions of a packed batch, to a window of the last tokens and the first few.

The Python binding of ``cb_attention_forward`` / ``_backward`` / ``_step`` (include/cb_tbe.h). Sessions
lie behind one another, named by offsets as the pooled calls' bags are; token t of a session that begins at s sees
token j, s <= j <= t, where t - j < window or j - s < sinks:

    out, lse = window_attention(q, k, v, offsets, window=256, sinks=4, stats=True)
    dq, dk, dv = window_attention_backward(grad_out, q, k, v, out, lse, offsets, window=256, sinks=4)
    out = window_attention_step(q, k_cache, v_cache, lengths, window=256, sinks=4)      # one new token each

Autograd records nothing of them: the second is the first's derivative, called by hand. fp16 and bf16
go through the tensor cores (heads of a multiple of 8 and at most 128 values), with sums, scores and softmax in
fp32; fp32 and other heads of up to 256 values go key by key, in fp32, and are far slower, over thousands of tokens in
sight than plain tensor operations would be. A row whose result is not finite is computed again that way, so a batch of
infinities costs as much. All work is enqueued on the current stream of the tensors' device; nothing waits.

``error``, everywhere: an int32 tensor of one value on the device, or None. A kernel sets it, if it holds 0, to the code of
what it met: offsets or lengths out of range, or (CB_ERR_TIMEOUT) a wait within it that ran out, after which results are
not whole. No input brings about the latter: it would be a fault of the library or the device.
"""

from __future__ import annotations

import ctypes

import torch

from . import tbe

# The entry points of include/cb_tbe.h that this module binds.
EXPORTS = ("cb_attention_forward", "cb_attention_backward", "cb_attention_workspace_bytes", "cb_attention_step",
           "cb_attention_step_workspace_bytes")

ALL = 2 ** 31 - 1  # a window that reaches every token

_bound = None


def _library() -> ctypes.CDLL:
    global _bound
    if _bound is None:
        lib = tbe.load_library()
        p, i32, i64, f32, c = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_int
        lib.cb_attention_forward.argtypes = [p, p, p, c, i64, i32, i32, i32, *[i64] * 6, p, c, i64, i64, i64, f32, p, i64,
                                             i64, p, p, i64, p, p]
        lib.cb_attention_backward.argtypes = [p, p, p, p, p, p, c, i64, i32, i32, i32, *[i64] * 10, p, c, i64, i64, i64, f32,
                                              p, p, p, *[i64] * 6, p, i64, p, p]
        lib.cb_attention_step.argtypes = [p, p, p, c, i64, i64, i32, i32, i32, *[i64] * 8, p, c, i64, i64, f32, p, i64, i64,
                                          p, i64, p, p]
        lib.cb_attention_workspace_bytes.argtypes = [i64, i32, i32, i32, i64, i64, c]
        lib.cb_attention_step_workspace_bytes.argtypes = [i64, i32, i32, i32, i64, i64, i64]
        for name in EXPORTS:
            getattr(lib, name).restype = i64 if name.endswith("bytes") else c
        _bound = lib
    return _bound


def _check_error(error: torch.Tensor, index: int):
    if error.get_device() != index or error.dtype != torch.int32 or error.numel() != 1:
        raise ValueError("error must be an int32 tensor of one value on the device")


def _index(t: torch.Tensor, what: str, index: int) -> int:
    kind = tbe._IDX.get(t.dtype)
    if kind is None or t.get_device() != index or t.dim() != 1 or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous, 1-D, int32 or int64 on the device of the other tensors")
    return kind


def _fits(t: torch.Tensor) -> bool:
    """Whether t's rows are contiguous and lie as the library's kernels for its type and size take them."""
    stride, dim = t.stride(), t.shape[-1]
    if dim > 1 and stride[-1] != 1:
        return False
    if t.dtype == torch.float32 or dim % 8 or dim > 128:
        return True
    return not (t.data_ptr() % 16 or any(s % 8 or s < dim for s, n in zip(stride[:-1], t.shape) if n > 1))  # TMA: 16 bytes


def _rows(t: torch.Tensor) -> torch.Tensor:
    return t if _fits(t) else t.clone(memory_format=torch.contiguous_format)


def _strides(t: torch.Tensor):
    """Strides of the leading dimensions, in values; a dimension of one has that of a whole row."""
    return [s if n > 1 else t.shape[-1] for s, n in zip(t.stride()[:-1], t.shape)]


def _shape(window, sinks, scale, dim: int):
    window = ALL if window is None else window
    if window < 1 or sinks < 0:
        raise ValueError("window must be at least 1 and sinks at least 0")
    return min(window, ALL), min(sinks, ALL), dim ** -0.5 if scale is None else scale


def _check_packed(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor):
    index = q.get_device()
    if index < 0 or q.dim() != 3 or k.dim() != 3:
        raise ValueError("q must be [tokens, heads, dim], k and v [tokens, kv_heads, dim], on a CUDA device")
    kind = tbe._DTYPES.get(q.dtype)
    if kind is None:
        raise ValueError(f"unsupported q dtype {q.dtype}")
    tokens, heads, dim = q.shape
    kv_heads = k.shape[1]
    for t in (k, v):
        if t.dtype != q.dtype or t.get_device() != index or t.shape != (tokens, kv_heads, dim):
            raise ValueError("k and v must be [tokens, kv_heads, dim] of q's type and device")
    if kv_heads < 1 or heads < 1 or heads % kv_heads:
        raise ValueError("the number of heads must be a multiple of that of k and v")
    if not 1 <= dim <= 256:
        raise ValueError("heads must have 1 to 256 values")
    return index, kind, tokens, heads, kv_heads, dim


def _output(out: torch.Tensor | None, like: torch.Tensor, what: str) -> torch.Tensor:
    if out is None:
        return torch.empty(like.shape, dtype=like.dtype, device=like.device)
    if out.shape != like.shape or out.dtype != like.dtype or out.get_device() != like.get_device():
        raise ValueError(f"{what} must be of shape {tuple(like.shape)}, type {like.dtype}, on the device")
    if out.shape[-1] > 1 and out.stride(-1) != 1:
        raise ValueError(f"{what} must have contiguous rows")
    return out


def window_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, offsets: torch.Tensor, window: int | None = None,
                     sinks: int = 0, scale: float | None = None, out: torch.Tensor | None = None, stats: bool = False,
                     error: torch.Tensor | None = None):
    """Attention of every token over its session (cb_attention_forward): out [tokens, heads, dim] in q's type.

    q: [tokens, heads, dim]; k, v: [tokens, kv_heads, dim]; slices of one projection's output are taken as they lie.
    offsets: int32 or int64 [sessions + 1]; tokens of no session give zeros. window None: all tokens before. scale:
    dim ** -0.5 unless given. out shares no memory with q, k, v. With stats=True the result is (out, lse), lse fp32
    [heads, tokens], as the backward pass takes it. error: set where offsets decrease or leave the tokens."""
    lib = _bound or _library()
    index, kind, tokens, heads, kv_heads, dim = _check_packed(q, k, v)
    off_kind = _index(offsets, "offsets", index)
    if offsets.numel() < 1:
        raise ValueError("offsets must hold at least one value")
    window, sinks, scale = _shape(window, sinks, scale, dim)
    if error is not None:
        _check_error(error, index)
    out = _output(out, q, "out")
    lse = torch.empty(heads, tokens, dtype=torch.float32, device=q.device) if stats else None
    if tokens:
        q, k, v = _rows(q), _rows(k), _rows(v)
        to = out if _fits(out) else torch.empty(out.shape, dtype=out.dtype, device=out.device)
        with tbe._OnDevice(index):
            nbytes = lib.cb_attention_workspace_bytes(tokens, heads, kv_heads, dim, window, sinks, 0)
            work = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
            status = lib.cb_attention_forward(
                q.data_ptr(), k.data_ptr(), v.data_ptr(), kind, tokens, heads, kv_heads, dim, *_strides(q), *_strides(k),
                *_strides(v), offsets.data_ptr(), off_kind, offsets.numel() - 1, window, sinks, scale, to.data_ptr(),
                *_strides(to), None if lse is None else lse.data_ptr(), work.data_ptr(), nbytes,
                None if error is None else error.data_ptr(), tbe._raw_stream(index))
        if status:
            tbe._check(status, "cb_attention_forward")
        if to is not out:
            out.copy_(to)
    return (out, lse) if stats else out


def window_attention_backward(grad_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                              lse: torch.Tensor, offsets: torch.Tensor, window: int | None = None, sinks: int = 0,
                              scale: float | None = None, grads=None, error: torch.Tensor | None = None):
    """The gradients (dq, dk, dv) of window_attention, from its inputs and its (out, lse) of stats=True
    (cb_attention_backward), in the inputs' type.

    grads: three tensors to write them to (slices of one buffer, say), which share no memory with the inputs or one
    another. error: as the forward pass."""
    lib = _bound or _library()
    index, kind, tokens, heads, kv_heads, dim = _check_packed(q, k, v)
    off_kind = _index(offsets, "offsets", index)
    if offsets.numel() < 1:
        raise ValueError("offsets must hold at least one value")
    window, sinks, scale = _shape(window, sinks, scale, dim)
    if error is not None:
        _check_error(error, index)
    for t, what in ((grad_out, "grad_out"), (out, "out")):
        if t.shape != q.shape or t.dtype != q.dtype or t.get_device() != index:
            raise ValueError(f"{what} must have q's shape, type and device")
    if lse.shape != (heads, tokens) or lse.dtype != torch.float32 or lse.get_device() != index:
        raise ValueError("lse must be fp32 [heads, tokens] on the device")
    given = (None, None, None) if grads is None else tuple(grads)
    if len(given) != 3:
        raise ValueError("grads must be three tensors")
    grads = tuple(_output(g, t, what) for g, t, what in zip(given, (q, k, v), ("dq", "dk", "dv")))
    if tokens:
        to = tuple(g if _fits(g) else torch.empty(g.shape, dtype=g.dtype, device=g.device) for g in grads)
        ins = [_rows(t) for t in (grad_out, q, k, v, out)]
        lse = lse.contiguous()
        with tbe._OnDevice(index):
            nbytes = lib.cb_attention_workspace_bytes(tokens, heads, kv_heads, dim, window, sinks, 1)
            work = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
            status = lib.cb_attention_backward(
                *[t.data_ptr() for t in ins], lse.data_ptr(), kind, tokens, heads, kv_heads, dim,
                *[s for t in ins for s in _strides(t)], offsets.data_ptr(), off_kind, offsets.numel() - 1, window, sinks, scale,
                *[t.data_ptr() for t in to], *[s for t in to for s in _strides(t)], work.data_ptr(), nbytes,
                None if error is None else error.data_ptr(), tbe._raw_stream(index))
        if status:
            tbe._check(status, "cb_attention_backward")
        for g, t in zip(grads, to):
            if g is not t:
                g.copy_(t)
    return grads


def window_attention_step(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, lengths: torch.Tensor,
                          window: int | None = None, sinks: int = 0, scale: float | None = None,
                          out: torch.Tensor | None = None, error: torch.Tensor | None = None) -> torch.Tensor:
    """Attention of one new token of each session, the last in its cache (cb_attention_step).

    q: [sessions, heads, dim]; k_cache, v_cache: [sessions, capacity, kv_heads, dim] in any strides with contiguous rows
    (a transposed [sessions, kv_heads, capacity, dim] too); lengths: int32 or int64 [sessions], the tokens of each,
    the new one among them, 0 .. capacity (0: zeros). out shares no memory with the inputs. Caches of halves whose addresses or
    strides are no multiples of 16 bytes go key by key, some 15 times slower. error: set to CB_ERR_INDEX_OOB by a length outside."""
    lib = _bound or _library()
    index = q.get_device()
    if index < 0 or q.dim() != 3 or k_cache.dim() != 4:
        raise ValueError("q must be [sessions, heads, dim], the caches [sessions, capacity, kv_heads, dim], on a CUDA device")
    kind = tbe._DTYPES.get(q.dtype)
    if kind is None:
        raise ValueError(f"unsupported q dtype {q.dtype}")
    sessions, heads, dim = q.shape
    capacity, kv_heads = k_cache.shape[1:3]
    for t in (k_cache, v_cache):
        if t.dtype != q.dtype or t.get_device() != index or t.shape != (sessions, capacity, kv_heads, dim):
            raise ValueError("the caches must be [sessions, capacity, kv_heads, dim] of q's type and device")
        if dim > 1 and t.stride(-1) != 1:
            raise ValueError("the caches' rows must be contiguous")
    if kv_heads < 1 or heads < 1 or heads % kv_heads or not 1 <= dim <= 256:
        raise ValueError("heads must be a multiple of kv_heads, and have 1 to 256 values")
    len_kind = _index(lengths, "lengths", index)
    if lengths.numel() != sessions:
        raise ValueError("lengths must hold a value for each session")
    window, sinks, scale = _shape(window, sinks, scale, dim)
    if error is not None:
        _check_error(error, index)
    out = _output(out, q, "out")
    if sessions:
        if dim > 1 and q.stride(-1) != 1:
            q = q.contiguous()
        with tbe._OnDevice(index):
            nbytes = lib.cb_attention_step_workspace_bytes(sessions, heads, kv_heads, dim, capacity, window, sinks)
            work = torch.empty(nbytes, dtype=torch.uint8, device=q.device) if nbytes else None
            status = lib.cb_attention_step(
                q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), kind, sessions, capacity, heads, kv_heads, dim,
                *_strides(q), *_strides(k_cache), *_strides(v_cache), lengths.data_ptr(), len_kind, window, sinks, scale,
                out.data_ptr(), *_strides(out), None if work is None else work.data_ptr(), nbytes,
                None if error is None else error.data_ptr(), tbe._raw_stream(index))
        if status:
            tbe._check(status, "cb_attention_step")
    return out
