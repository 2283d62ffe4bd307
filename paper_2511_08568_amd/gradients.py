"""Norm of many gradients together, and their clipping.

    norm = clip_grad_norm(grads, max_norm)             # in place
    grads = GradientList(grads, out=master_grads)      # kept from step to step
    norm = clip_grad_norm(grads, max_norm)             # clipped copies in master_grads

The functions check and pass on their arguments; nothing here computes.  They
enqueue on ``stream`` (default: the current stream of the tensors' device) and do
not synchronise; the norm is a tensor on the device.  Work that makes their
tensors has to be waited for by ``stream``; the tensors may be dropped at once.
"""
from __future__ import annotations

import bisect
import ctypes
import functools

import torch

from . import binding as bd
from .embedding import DTYPES, _current_stream, _dual, _elsewhere, _Switch, _tangents, _written

_workspace_bytes = functools.lru_cache(maxsize=256)(bd.recmg_query_grad_workspace)


def _dense(t) -> bool:
    """Whether the tensor's elements fill one range of memory, each place once."""
    if t.is_contiguous():
        return True
    want = 1
    for size, stride in sorted(((s, st) for s, st in zip(t.shape, t.stride()) if s != 1), key=lambda x: x[1]):
        if stride != want:
            return False
        want *= size
    return True


class GradientList:
    """The gradients of a step, laid out once for grad_norm, clip_grads and
    clip_grad_norm.  It stands for the memory that the tensors have then, holds it,
    and refuses calls once that memory has been resized (``resize_`` beyond its end).
    Build it again when a gradient is another tensor, of another size, or has been
    given other memory (``.data =``, ``set_``): the calls take the former memory.

    grads: cuda tensors (float32 / float16 / bfloat16, each filling one range of
    memory, all on one device), or pairs (values, count) of embedding_backward_rows,
    of which the first count rows take part.  out: where clipped gradients go, a
    tensor per gradient of its shape and strides and of any of the three types;
    without it they are clipped in place."""

    def __init__(self, grads, out=None):
        self.tensors, self.counts = [], []
        for g in grads:
            values, count = g if isinstance(g, (tuple, list)) else (g, None)
            if count is not None:
                if values.dim() != 2 or not values.is_contiguous():
                    raise ValueError("values with a count must be a contiguous matrix")
                if values.shape[1] >= 1 << 31:  # ctypes would cut it to 32 bits
                    raise ValueError("values with a count: fewer than 2^31 columns")
                if count.dtype != torch.int64 or count.numel() != 1 or count.device != values.device:
                    raise ValueError("count: one int64 on the device of its values")
            self.tensors.append(values)
            self.counts.append(count)
        n = self.n = len(self.tensors)
        self.outs = self.tensors if out is None else list(out)
        if len(self.outs) != n:
            raise ValueError(f"out: {n} tensors, one per gradient, not {len(self.outs)}")
        self.device = self.tensors[0].device if n else None
        for t in self.tensors + ([] if out is None else self.outs):
            if not t.is_cuda or t.dtype not in DTYPES:
                raise ValueError("gradients are float32, float16 or bfloat16 tensors on the GPU")
            if t.device != self.device:
                raise ValueError(f"gradients on {self.device} and on {t.device}")
            if not _dense(t):
                raise ValueError("a gradient must fill one range of memory")
        for g, o in zip(self.tensors, self.outs):
            if o is not g and (o.shape != g.shape or (o.stride() != g.stride() and not (o.is_contiguous() and g.is_contiguous()))):
                raise ValueError("an output must have its gradient's shape and strides")
        some = max(n, 1)
        self._grads = (ctypes.c_void_p * some)(*[t.data_ptr() for t in self.tensors])
        self._outs = (ctypes.c_void_p * some)(*[t.data_ptr() for t in self.outs])
        self._numels = (ctypes.c_int64 * some)(*[t.numel() for t in self.tensors])
        self._dtypes = (ctypes.c_int32 * some)(*[DTYPES[t.dtype] for t in self.tensors])
        self._out_dtypes = (ctypes.c_int32 * some)(*[DTYPES[t.dtype] for t in self.outs])
        self._live = self._lengths = None
        if any(c is not None for c in self.counts):
            self._live = (ctypes.c_void_p * some)(*[None if c is None else c.data_ptr() for c in self.counts])
            self._lengths = (ctypes.c_int32 * some)(*[0 if c is None else max(1, t.shape[1])
                                                      for c, t in zip(self.counts, self.tensors)])
        self._apart = False
        # a tensor and its views count their changes together
        self._counting = list({id(t): t for t in (t if t._base is None else t._base for t in self.outs)}.values())
        # the storages behind the addresses that the calls use: held, so that no other tensor comes to lie there
        held = self.tensors + ([] if out is None else self.outs) + [c for c in self.counts if c is not None]
        self._memory = list({s.data_ptr(): s for s in (t.untyped_storage() for t in held)}.values())
        self._like = self.tensors[0].detach() if n else None  # what results are made like: not the caller's to change
        self._places = [(s.data_ptr(), s.nbytes()) for s in self._memory]

    def _check_memory(self):
        """A resized storage has let its memory go.  (62 tensors with a storage each: 12.4 us of the host per call
        without this, 17.6 with it; views of one buffer: no difference.)"""
        if [(s.data_ptr(), s.nbytes()) for s in self._memory] != self._places:
            raise ValueError("a tensor's memory has been resized: build the GradientList again")

    def _bytes(self):
        """The list's memory as tensors, whatever its own tensors are by now."""
        return [self._like.new_empty(0, dtype=torch.uint8).set_(s) for s in self._memory]

    def _check_apart(self):
        """Outputs share memory with nothing but their own gradients."""
        if self._apart:
            return
        spans = lambda at, types: [(p or 0, (p or 0) + self._numels[k] * (4 if types[k] == bd.RECMG_F32 else 2))  # noqa: E731
                                   for k, p in enumerate(at[:self.n])]
        outs = sorted((*span, k) for k, span in enumerate(spans(self._outs, self._out_dtypes)) if self._numels[k])
        for a, b in zip(outs, outs[1:]):
            if b[0] < a[1]:
                raise ValueError(f"outputs {a[2]} and {b[2]} share memory: each gradient may be clipped once")
        starts = [o[0] for o in outs]
        for k, (lo, hi) in enumerate(spans(self._grads, self._dtypes)):
            at = bisect.bisect_right(starts, lo) - 1
            for start, end, j in outs[max(at, 0):bisect.bisect_left(starts, hi)] if lo < hi else []:
                if start < hi and lo < end and not (j == k and start == lo and end == hi):
                    raise ValueError(f"output {j} shares memory with gradient {k}")
        self._spans, self._starts = outs, starts
        for k, c in enumerate(self.counts):
            if c is not None:
                self._check_scalar(f"count {k}", self._live[k], 8)
        self._apart = True

    def _check_scalar(self, name, at, size):
        """Outputs share no memory with a count or the norm, which all blocks of the clipping read."""
        k = bisect.bisect_left(self._starts, at + size) - 1
        if k >= 0 and self._spans[k][1] > at:
            raise ValueError(f"output {self._spans[k][2]} shares memory with {name}")


def _list(grads, out=None) -> GradientList:
    if isinstance(grads, GradientList):
        if out is not None:
            raise ValueError("a GradientList has its outputs already")
        grads._check_memory()
        return grads
    return GradientList(grads, out=out)


def _call(g: GradientList, stream, norm, max_norm, eps):
    """The norm (if `norm` is None) and the clipping (if `max_norm` is not), on `stream`."""
    if g.n == 0:
        raise ValueError("no gradients")
    if _tangents._current_level >= 0 and any(map(_dual, [*g.tensors, *g.outs])):
        raise ValueError("a gradient has a tangent, which this call would not pass on")
    if _elsewhere(g.device, stream):
        with _Switch(g.device, stream, (norm, *g._bytes())):
            return _call(g, None, norm, max_norm, eps)
    lib, s = bd.load_library(), _current_stream(g.device.index)
    if norm is not None:
        status = lib.recmg_grad_clip(g.n, g._grads, g._outs, g._numels, g._dtypes, g._out_dtypes, g._live, g._lengths,
                                     norm.data_ptr(), max_norm, eps, s)
    else:
        size = _workspace_bytes(g.n)
        norm, work = g._like.new_empty((), dtype=torch.float32), g._like.new_empty(size, dtype=torch.uint8)
        if max_norm is None:
            status = lib.recmg_grad_norm(g.n, g._grads, g._numels, g._dtypes, g._live, g._lengths, norm.data_ptr(),
                                         work.data_ptr(), size, s)
        else:
            status = lib.recmg_grad_norm_clip(g.n, g._grads, g._outs, g._numels, g._dtypes, g._out_dtypes, g._live,
                                              g._lengths, norm.data_ptr(), max_norm, eps, work.data_ptr(), size, s)
    if status:
        bd._check(status, "recmg_grad_norm_clip" if max_norm is not None else "recmg_grad_norm")
    if max_norm is not None:
        _written(g._counting)
    return norm


def grad_norm(grads, *, stream=None):
    """sqrt of the sum of squares over all gradients: a float32 tensor of no
    dimension on their device.  grads: a GradientList, or what one is made of."""
    return _call(_list(grads), stream, None, None, 0.0)


def clip_grads(grads, norm, max_norm: float, *, out=None, eps: float = 1e-6, stream=None):
    """Multiplies all gradients by min(1, max_norm / (norm + eps)), by 0 if norm is
    infinite, in place or into the outputs.  norm: one float32 on their device, from
    grad_norm (or the norm over several processes' gradients, made of theirs)."""
    g = _list(grads, out)
    if norm.dtype != torch.float32 or norm.numel() != 1 or norm.device != g.device:
        raise ValueError(f"norm: one float32 on {g.device}")
    g._check_apart()
    g._check_scalar("the norm", norm.data_ptr(), 4)
    _call(g, stream, norm, max_norm, eps)


def clip_grad_norm(grads, max_norm: float, *, out=None, eps: float = 1e-6, stream=None):
    """grad_norm, then clip_grads with the norm in 64 bits; returns the norm before
    clipping."""
    g = _list(grads, out)
    g._check_apart()
    return _call(g, stream, None, max_norm, eps)
