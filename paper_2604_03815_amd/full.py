"""Full softmax attention over packed sequences: front end of kmip_full_fwd / kmip_full_bwd.

The dense counterpart of ``attention``: every key of a query's sequence (or
graph) is kept.  Tensors: q [Nq, H, d], k_ [Nk, Hk, d] and v [Nk, Hk, dv] in
bfloat16 or float16, H a multiple of Hk (query head h reads key head
h // (H // Hk)); widths in {16, 32, 64, 128}.  out [Nq, H, dv] and the gradients have the inputs' type,
lse is float32 [Nq, H].  q, k_, v and dout may be views whose last dimension is
contiguous and whose other strides are multiples of 8 values, such as slices of
one fused projection; outputs are contiguous.

Sequences: ``graph_offsets`` (host int sequence [G+1]) cuts the rows of q;
``key_offsets`` those of k_ and v (None: the same); ``key_lengths`` (host [G]) says
how many keys at the start of each slot are in use (None: all), for caches
with room.  Without graph_offsets there is one sequence.  ``causal``: the queries are the
last positions of their sequence, query t of m sees keys 0 .. t + n - m of n.
The offsets and lengths are read when the call is made: a captured call keeps them.
Inputs are finite (rows behind the keys in use may hold anything: they are not read);
given outputs overlap neither inputs nor each other, and require no gradient (unless under torch.no_grad()).  A call's sequences are cut into jobs alike: single tokens over long
caches and long prompts are faster in calls of their own.
"""
from __future__ import annotations

import array
import ctypes
import functools
from typing import Optional, Sequence

import numpy as np
import torch

from ._lib import BF16, FP16, FP32, FULL_LONG, check, load

_DTYPES = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32}
_HALF = {torch.bfloat16: BF16, torch.float16: FP16}


def _check_tensor(t, name, dtype, shape):
    """A tensor of this type and shape whose last dimension is contiguous; whether all of it is."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.is_contiguous():
        return True
    if t.shape[-1] > 1 and t.stride(-1) != 1 and t.numel():
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return False


def _check_written(t, name):
    """A tensor to write into is no part of a graph of autograd's, which would go on with the gradient of its old values."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient: writing into it is not differentiable, call under torch.no_grad()")


def _check_output(t, name, dtype, shape):
    if t is None:
        return
    if not _check_tensor(t, name, dtype, shape):
        raise ValueError(f"{name} must be contiguous")
    _check_written(t, name)


def _new(like, shape, dtype):
    """A contiguous tensor of this shape and type on like's device (the cheapest way to it)."""
    if like.shape == shape and like.dtype == dtype:
        return torch.empty_like(like, memory_format=torch.contiguous_format)
    return like.new_empty(shape, dtype=dtype)


def _strides(*tensors):
    """Host int64 pairs of strides (0 for a dimension of one, whose stride can be anything)."""
    s = [x if n > 1 else 0 for t in tensors for n, x in zip(t.shape[:2], t.stride())]
    return (ctypes.c_int64 * len(s))(*s)


def _check_devices(*named):
    dev = named[0][0].device
    for t, name in named:
        if t is None:
            continue
        if not t.is_cuda:
            raise TypeError(f"{name} must be a CUDA (HIP) tensor")
        if t.device != dev:
            raise ValueError(f"{name} is on {t.device}, expected {dev} (the device of {named[0][1]})")
    return dev


def _written(*given):
    """The caller's own tensors among these were written: autograd, which the launch went past, counts it like an operation of torch's."""
    given = [t for t in given if t is not None]
    if given:
        torch.autograd.graph.increment_version(given)


def _launch(device, call, *args):
    """call(*args, stream) with the tensors' device current, on its current stream."""
    i = device.index
    if torch._C._cuda_getDevice() == i:
        check(call(*args, torch._C._cuda_getCurrentRawStream(i)))
    else:
        with torch.cuda.device(device):
            check(call(*args, torch._C._cuda_getCurrentRawStream(i)))


class _Ints:
    """A host int32 array of a 1-D integer sequence, and its address."""

    __slots__ = ("keep", "ptr", "count", "most")

    def __init__(self, values, name, n=None):
        try:
            if isinstance(values, (list, tuple)):
                a = array.array("i", values)
                self.ptr, self.count = a.buffer_info()
            else:
                a = np.asarray(values)
                if a.ndim != 1 or a.dtype.kind not in "iu":
                    raise TypeError
                if a.size and (int(a.min()) < -(1 << 31) or int(a.max()) >= 1 << 31):
                    raise OverflowError
                a = np.ascontiguousarray(a, dtype=np.int32)
                self.ptr, self.count = a.__array_interface__["data"][0], len(a)
        except (TypeError, OverflowError):
            raise ValueError(f"{name} must be a 1-D sequence of 32-bit integers") from None
        if self.count < 2 if n is None else self.count != n:
            raise ValueError(f"{name} must have {'at least two' if n is None else n} entries, got {self.count}")
        self.keep = a


def _sequences(graph_offsets, key_offsets, key_lengths):
    """Host arrays (to be kept alive over the call), their addresses, the number of sequences."""
    qo = None if graph_offsets is None else _Ints(graph_offsets, "graph_offsets")
    G = 1 if qo is None else qo.count - 1
    if qo is None and key_offsets is not None:
        raise ValueError("key_offsets needs graph_offsets")
    ko = None if key_offsets is None else _Ints(key_offsets, "key_offsets", G + 1)
    kl = None if key_lengths is None else _Ints(key_lengths, "key_lengths", G)
    return (qo, ko, kl), tuple(None if a is None else a.ptr for a in (qo, ko, kl)), G


def _inputs(q, k_, v):
    """Checks Q, K and V; returns (Nq, Nk, H, Hk, d, dv), the dtype's code and whether all are contiguous."""
    for t, name in ((q, "Q"), (k_, "K"), (v, "V")):
        if not isinstance(t, torch.Tensor) or t.dim() != 3:
            raise ValueError(f"{name} must be a tensor [N, heads, width]")
    dtype = q.dtype
    code = _HALF.get(dtype)
    if code is None:
        raise TypeError(f"Q must be torch.bfloat16 or torch.float16, got {dtype}")
    Nq, H, d = q.shape
    Nk, Hk, dv = v.shape
    whole = _check_tensor(q, "Q", dtype, (Nq, H, d))
    whole &= _check_tensor(k_, "K", dtype, (Nk, Hk, d))
    whole &= _check_tensor(v, "V", dtype, (Nk, Hk, dv))
    return (Nq, Nk, H, Hk, d, dv), code, whole


def _scratch(workspace, nbytes, device):
    if nbytes == 0:
        return None
    # (a captured call keeps its addresses: it gets memory of its own, which no later call grows or shares)
    if workspace is None or torch.cuda.is_current_stream_capturing():
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    buf = workspace.get(nbytes)
    if buf.device != device:
        raise ValueError(f"workspace is on {buf.device}, expected {device}")
    return buf


def _address(t):
    return None if t is None else t.data_ptr()


def full_fwd_workspace_size(Nq: int, Nk: int, H: int, Hk: int, d: int, dv: int, graph_offsets=None, key_offsets=None,
                            key_lengths=None) -> int:
    keep, ptrs, G = _sequences(graph_offsets, key_offsets, key_lengths)
    return int(load().kmip_full_fwd_workspace_size(*ptrs, G, Nq, Nk, H, Hk, d, dv))


def full_fwd(q, k_, v, scale: float, graph_offsets: Optional[Sequence[int]] = None, key_offsets=None, key_lengths=None,
             causal: bool = False, out=None, lse=None, workspace=None):
    """Full softmax attention: returns (out, lse)."""
    sizes, code, whole = _inputs(q, k_, v)
    Nq, Nk, H, Hk, d, dv = sizes
    _check_output(out, "out", q.dtype, (Nq, H, dv))
    _check_output(lse, "lse", torch.float32, (Nq, H))
    keep, ptrs, G = _sequences(graph_offsets, key_offsets, key_lengths)
    dev = _check_devices((q, "Q"), (k_, "K"), (v, "V"), (out, "out"), (lse, "lse"))
    lib = load()
    given = out, lse
    buf = None
    if Nk >= FULL_LONG:
        buf = _scratch(workspace, lib.kmip_full_fwd_workspace_size(*ptrs, G, *sizes), dev)
    if out is None:
        out = _new(q, (Nq, H, dv), q.dtype)
    if lse is None:
        lse = q.new_empty((Nq, H), dtype=torch.float32)
    _launch(dev, lib.kmip_full_fwd, q.data_ptr(), k_.data_ptr(), v.data_ptr(), code, None if whole else _strides(q, k_, v), *ptrs, G,
            *sizes, float(scale), 1 if causal else 0, out.data_ptr(), lse.data_ptr(), _address(buf), 0 if buf is None else buf.numel())
    _written(*given)
    return out, lse


def full_bwd_workspace_size(Nq: int, Nk: int, H: int, Hk: int, d: int, dv: int, graph_offsets=None, key_offsets=None,
                            key_lengths=None) -> int:
    keep, ptrs, G = _sequences(graph_offsets, key_offsets, key_lengths)
    return int(load().kmip_full_bwd_workspace_size(*ptrs, G, Nq, Nk, H, Hk, d, dv))


def full_bwd(q, k_, v, dout, out, lse, scale: float, graph_offsets: Optional[Sequence[int]] = None, key_offsets=None,
             key_lengths=None, causal: bool = False, dq=None, dk=None, dv=None, workspace=None):
    """Gradients of full softmax attention: returns (dQ, dK, dV) of the inputs' type."""
    sizes, code, whole = _inputs(q, k_, v)
    Nq, Nk, H, Hk, d, wv = sizes
    whole &= _check_tensor(dout, "dOut", q.dtype, (Nq, H, wv))
    for t, name, dtype, shape in ((out, "out", q.dtype, (Nq, H, wv)), (lse, "lse", torch.float32, (Nq, H))):
        if not _check_tensor(t, name, dtype, shape):
            raise ValueError(f"{name} must be contiguous")
    _check_output(dq, "dQ", q.dtype, (Nq, H, d))
    _check_output(dk, "dK", q.dtype, (Nk, Hk, d))
    _check_output(dv, "dV", q.dtype, (Nk, Hk, wv))
    keep, ptrs, G = _sequences(graph_offsets, key_offsets, key_lengths)
    dev = _check_devices((q, "Q"), (k_, "K"), (v, "V"), (dout, "dOut"), (out, "out"), (lse, "lse"), (dq, "dQ"), (dk, "dK"),
                         (dv, "dV"))
    lib = load()
    given = dq, dk, dv
    buf = _scratch(workspace, lib.kmip_full_bwd_workspace_size(*ptrs, G, *sizes), dev)
    if dq is None:
        dq = _new(q, (Nq, H, d), q.dtype)
    if dk is None:
        dk = _new(k_, (Nk, Hk, d), q.dtype)
    if dv is None:
        dv = _new(v, (Nk, Hk, wv), q.dtype)
    _launch(dev, lib.kmip_full_bwd, q.data_ptr(), k_.data_ptr(), v.data_ptr(), dout.data_ptr(), out.data_ptr(), lse.data_ptr(),
            code, None if whole else _strides(q, k_, v, dout), *ptrs, G, *sizes, float(scale), 1 if causal else 0, dq.data_ptr(), dk.data_ptr(),
            dv.data_ptr(), _address(buf), 0 if buf is None else buf.numel())
    _written(*given)
    return dq, dk, dv


def full_attention(q, k_, v, scale: float, graph_offsets: Optional[Sequence[int]] = None, key_offsets=None,
                   key_lengths=None, causal: bool = False, workspace=None):
    """Differentiable full softmax attention: returns out [Nq, H, dv] of the inputs' type.

    The forward is ``full_fwd``; autograd's backward calls ``full_bwd`` with
    the saved out and lse.  Once differentiable.  To capture a backward into a
    HIP graph, run it on a side stream first, and let go of every eager result of
    the same leaves: autograd ties a leaf's gradient to the stream of the first.
    """
    # (copies: the caller may change its own before the backward)
    where = {n: None if x is None else np.array(x) for n, x in (("graph_offsets", graph_offsets), ("key_offsets", key_offsets),
                                                                ("key_lengths", key_lengths))}
    where["causal"] = causal
    return _full_function().apply(q, k_, v, scale, where, workspace)


@functools.lru_cache(maxsize=None)
def _full_function():
    class _Full(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k_, v, scale, where, workspace):
            out, lse = full_fwd(q, k_, v, scale, workspace=workspace, **where)
            ctx.save_for_backward(q, k_, v, out, lse)
            ctx.args = scale, where, workspace
            return out

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dout):
            q, k_, v, out, lse = ctx.saved_tensors
            scale, where, workspace = ctx.args
            if dout.stride(-1) != 1 or any(s % 8 for s in dout.stride()[:2]) or dout.stride(0) >= 1 << 23 or dout.data_ptr() % 16:
                dout = dout.contiguous()
            return (*full_bwd(q, k_, v, dout, out, lse, scale, workspace=workspace, **where), None, None, None)

    return _Full
