"""Lookup of token ids in a table that device memory holds, and the gradient of
lookups: for the whole table, or as its distinct rows.

    x = embedding_forward(table, tokens, scale=...)
    grad = embedding_backward(grad_x, tokens, rows, scale=...)
    rows, values, count = embedding_backward_rows(grad_x, tokens, rows, ...)

With ``offsets`` the gradient is that of the pooled sum of
``TieredEmbeddingCache.forward`` for one table.  The functions check and pass on
their arguments; nothing here computes.  They enqueue on ``stream`` (default: the
current stream of the tensors' device), allocate results and workspaces there,
and do not synchronise.  Work that makes their tensors has to be waited for by
``stream``; the tensors may be dropped at once.  Autograd does not record them:
while it is enabled, tensors that require a gradient are refused, and those with
a forward-mode tangent always.
"""
from __future__ import annotations

import functools
import types

import torch
from torch.autograd import forward_ad

from . import binding as bd

DTYPES = {torch.float32: bd.RECMG_F32, torch.float16: bd.RECMG_F16, torch.bfloat16: bd.RECMG_BF16}
INDEX_TYPES = {torch.int32: bd.RECMG_I32, torch.int64: bd.RECMG_I64}

_workspace_bytes = functools.lru_cache(maxsize=256)(bd.recmg_query_embedding_workspace)


# the current stream's handle (the public call makes a stream object first, which takes as long as a launch) and device
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
# marks a list's tensors as changed, so that autograd sees values that it has kept for a backward pass written over
_written = getattr(torch._C, "_increment_version", None) or torch.autograd.graph.increment_version
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


class _Switch:
    """Makes a stream (or a device alone) current for a call, and records that the stream uses `tensors`: their memory
    goes to nobody else before the call's kernels have ended, also where the caller drops them at once."""

    __slots__ = ("guard", "stream", "tensors")

    def __init__(self, device, stream, tensors):
        if stream is not None and stream.device != device:
            raise ValueError(f"stream is on {stream.device}, the tensors on {device}")
        self.guard = torch.cuda.stream(stream) if stream is not None else torch.cuda.device(device)
        self.stream, self.tensors = stream, tensors

    def __enter__(self):
        return self.guard.__enter__()

    def __exit__(self, kind, *exc):
        self.guard.__exit__(kind, *exc)
        if kind is None and self.stream is not None:
            for t in self.tensors:
                if t is not None:
                    t.record_stream(self.stream)


def _elsewhere(device, stream) -> bool:
    """Whether a call on `stream` (None: the current one) of `device` needs a _Switch: results and workspaces come from
    the current stream's memory, and kernels go to the current device."""
    return device.type == "cuda" and (stream is not None or device.index != _current_device())


# the level of forward-mode tangents, below 0 outside them all (where torch does not say, every tensor is asked)
_tangents = forward_ad if hasattr(forward_ad, "_current_level") else types.SimpleNamespace(_current_level=0)


def _dual(t) -> bool:
    return forward_ad.unpack_dual(t).tangent is not None


def _unrecorded(name: str, t):
    """Refuses what autograd would have to record."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, but autograd does not record this call: pass {name}.detach()")
    if _tangents._current_level >= 0 and _dual(t):
        raise ValueError(f"{name} has a tangent, which this call would not pass on")


def _matrix(name: str, t, least_stride_is_dim: bool = True):
    """(address, dtype code, row stride) of a matrix of rows of adjacent elements."""
    shape = t.shape
    if len(shape) != 2 or not t.is_cuda:
        raise ValueError(f"{name} must be a 2-D tensor on the GPU")
    code = DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: float32, float16 or bfloat16, not {t.dtype}")
    n, dim = shape
    stride, step = t.stride()
    if dim > 1 and step != 1:
        raise ValueError(f"{name}: the elements of a row must be adjacent")
    if dim >= 1 << 31:  # ctypes would cut it to 32 bits
        raise ValueError(f"{name}: at most 65536 columns, not {dim}")
    if n <= 1:
        stride = dim
    elif least_stride_is_dim and stride < dim:
        raise ValueError(f"{name}: rows overlap")
    return t.data_ptr(), code, stride


def _id(name: str, value: int):
    """ctypes would cut a larger number to 64 bits."""
    if not -(1 << 63) <= value < 1 << 63:
        raise ValueError(f"{name} is no 64-bit number")


def _ids(name: str, t, device):
    code = INDEX_TYPES.get(t.dtype)
    if code is None or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous int32 or int64")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    return t.data_ptr(), code, t.numel()


def embedding_forward(table, tokens, *, scale: float = 1.0, first_row: int = 0, out=None, out_dtype=None, stream=None):
    """scale * table[tokens - first_row], of shape tokens.shape + (dim,).

    table: cuda [rows, dim], float32 / float16 / bfloat16 (rows may be strided, as
    in a slice of columns).  tokens: cuda int32 or int64 of any shape, contiguous;
    a token outside [first_row, first_row + rows) gives zeros.  out: a tensor
    [tokens.numel(), dim] to write into; out_dtype: the table's by default."""
    device = table.device
    if _elsewhere(device, stream):
        with _Switch(device, stream, (table, tokens, out)):
            return embedding_forward(table, tokens, scale=scale, first_row=first_row, out=out, out_dtype=out_dtype)
    _unrecorded("table", table)
    if first_row:
        _id("first_row", first_row)
    ptr, code, stride = _matrix("table", table)
    rows, dim = table.shape
    ids, index_type, n = _ids("tokens", tokens, device)
    written = out is not None
    if not written:
        if out_dtype is None:
            out, o_code = table.new_empty((*tokens.shape, dim)), code
        else:
            o_code = DTYPES.get(out_dtype)
            if o_code is None:
                raise ValueError(f"out_dtype: float32, float16 or bfloat16, not {out_dtype}")
            out = table.new_empty((*tokens.shape, dim), dtype=out_dtype)
        o_ptr, o_stride = out.data_ptr(), dim
    else:
        _unrecorded("out", out)
        if out.device != device or out.shape != (n, dim) or out_dtype not in (None, out.dtype):
            raise ValueError(f"out must be [{n}, {dim}] on {device}, of out_dtype if that is given")
        o_ptr, o_code, o_stride = _matrix("out", out)
    status = bd.load_library().recmg_embedding_forward(ptr, code, stride, rows, dim, ids, index_type, n, first_row, scale,
                                                       o_ptr, o_code, o_stride, _current_stream(device.index))
    if status:
        bd._check(status, "recmg_embedding_forward")
    if written:
        _written([out])
    return out


def _given(grad_out, tokens, offsets, rows, first_row, padding_token):
    """The arguments that both forms of the gradient share, checked: what the C entries take of them."""
    if not 0 < rows < 1 << 31:
        raise ValueError("rows: 1 to 2^31 - 1")
    _id("first_row", first_row)
    _id("padding_token", padding_token)
    _unrecorded("grad_out", grad_out)
    ptr, code, stride = _matrix("grad_out", grad_out, least_stride_is_dim=False)
    device = grad_out.device
    ids, index_type, n = _ids("tokens", tokens, device)
    if offsets is None:
        if grad_out.shape[0] != n:
            raise ValueError(f"grad_out has {grad_out.shape[0]} rows for {n} tokens")
        return device, n, (ptr, code, stride, ids, index_type, n, None, 0)
    if offsets.dtype != torch.int64 or offsets.dim() != 1 or not offsets.is_contiguous() or offsets.device != device \
            or offsets.numel() != grad_out.shape[0] + 1:
        raise ValueError(f"offsets must be int64 [{grad_out.shape[0] + 1}] on {device}, one more than grad_out has rows")
    return device, n, (ptr, code, stride, ids, index_type, n, offsets.data_ptr(), grad_out.shape[0])


def embedding_backward(grad_out, tokens, rows: int, *, offsets=None, scale: float = 1.0, first_row: int = 0,
                       padding_token: int = -1, grad=None, accumulate: bool = False, dtype=None, stream=None):
    """Gradient [rows, dim] of embedding_forward with respect to its table.

    grad_out: cuda [tokens.numel(), dim], or with offsets [bags, dim] (rows may be
    strided, or one row expanded).  offsets: cuda int64 [bags + 1], the bags of the
    tokens; offsets[0] is where the first token lies in its batch.  padding_token
    (or None): an id without a gradient.  grad: written whole, or added to with
    accumulate; else a new tensor of `dtype` (default: grad_out's)."""
    if _elsewhere(grad_out.device, stream):
        with _Switch(grad_out.device, stream, (grad_out, tokens, offsets, grad)):
            return embedding_backward(grad_out, tokens, rows, offsets=offsets, scale=scale, first_row=first_row,
                                      padding_token=padding_token, grad=grad, accumulate=accumulate, dtype=dtype)
    padding_token = -1 if padding_token is None else padding_token
    device, n, given = _given(grad_out, tokens, offsets, rows, first_row, padding_token)
    dim = grad_out.shape[1]
    written = grad is not None
    if not written:
        if accumulate:
            raise ValueError("accumulate needs the gradient to add to (grad)")
        grad = grad_out.new_empty((rows, dim), dtype=dtype)
    elif grad.device != device or grad.shape != (rows, dim) or dtype not in (None, grad.dtype):
        raise ValueError(f"grad must be [{rows}, {dim}] on {device}, of dtype if that is given")
    _unrecorded("grad", grad)
    ptr, code, stride = _matrix("grad", grad)
    size = _workspace_bytes(rows, dim, n, 0, offsets is not None)
    work = grad_out.new_empty(size, dtype=torch.uint8) if size else None
    status = bd.load_library().recmg_embedding_backward(
        *given, rows, dim, first_row, padding_token, scale, ptr, code, stride,
        bool(accumulate), work.data_ptr() if size else None, size, _current_stream(device.index))
    if status:
        bd._check(status, "recmg_embedding_backward")
    if written:
        _written([grad])
    return grad


def embedding_backward_rows(grad_out, tokens, rows: int, *, offsets=None, scale: float = 1.0, first_row: int = 0,
                            padding_token: int = -1, out=None, dtype=None, stream=None):
    """The same gradient as (row numbers, values, count): the distinct rows that
    tokens name, ascending (int32, tokens - first_row), their gradients, and how many
    they are (int64 [1], on the device).  Both hold min(tokens.numel(), rows) rows;
    what lies behind the count is left as it was.  out: the three tensors to write
    into; else new ones, the values of `dtype` (default float32)."""
    if _elsewhere(grad_out.device, stream):
        with _Switch(grad_out.device, stream, (grad_out, tokens, offsets, *(out or ()))):
            return embedding_backward_rows(grad_out, tokens, rows, offsets=offsets, scale=scale, first_row=first_row,
                                           padding_token=padding_token, out=out, dtype=dtype)
    padding_token = -1 if padding_token is None else padding_token
    device, n, given = _given(grad_out, tokens, offsets, rows, first_row, padding_token)
    dim = grad_out.shape[1]
    cap = min(n, rows)
    written = out is not None
    if not written:
        out = (grad_out.new_empty(cap, dtype=torch.int32), grad_out.new_empty((cap, dim), dtype=dtype or torch.float32),
               grad_out.new_empty(1, dtype=torch.int64))
    number, values, count = out
    if number.device != device or number.dtype != torch.int32 or not number.is_contiguous() or number.numel() < cap:
        raise ValueError(f"row numbers: contiguous int32 of at least {cap} on {device}")
    if values.device != device or values.dim() != 2 or values.shape[1] != dim or values.shape[0] < cap \
            or dtype not in (None, values.dtype):
        raise ValueError(f"values: at least {cap} rows of {dim} on {device}, of dtype if that is given")
    if count.device != device or count.dtype != torch.int64 or count.numel() != 1:
        raise ValueError(f"count: one int64 on {device}")
    _unrecorded("values", values)
    ptr, code, stride = _matrix("values", values)
    size = _workspace_bytes(rows, dim, n, 1, offsets is not None)
    work = grad_out.new_empty(size, dtype=torch.uint8) if size else None
    status = bd.load_library().recmg_embedding_backward_rows(
        *given, rows, dim, first_row, padding_token, scale, number.data_ptr(), ptr, code,
        stride, count.data_ptr(), work.data_ptr() if size else None, size, _current_stream(device.index))
    if status:
        bd._check(status, "recmg_embedding_backward_rows")
    if written:
        _written([number, values, count])
    return out
