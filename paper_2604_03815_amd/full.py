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
"""
from __future__ import annotations

import ctypes
import functools
from typing import Optional, Sequence

import numpy as np
import torch

from ._lib import BF16, FP16, FP32, check, load

_DTYPES = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32}


def _ptr(t):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


def _check_view(t, name, dtype, shape):
    """A tensor of this type and shape whose last dimension is contiguous; returns its two other strides in values."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.numel() and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return t.stride(0), t.stride(1)


def _check_devices(*named):
    dev = named[0][0].device
    for t, name in named:
        if not t.is_cuda:
            raise TypeError(f"{name} must be a CUDA (HIP) tensor")
        if t.device != dev:
            raise ValueError(f"{name} is on {t.device}, expected {dev} (the device of {named[0][1]})")
    return dev


class _on_device:
    """The device of the tensors as the current one while a call launches, and its current stream."""

    def __init__(self, device):
        self.guard = torch.cuda.device(device) if torch.cuda.current_device() != device.index else None

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _int32(values, name, n=None):
    a = np.asarray(values)
    if a.ndim != 1 or a.dtype.kind not in "iu" or (n is not None and len(a) != n) or (n is None and len(a) < 2):
        raise ValueError(f"{name} must be a 1-D integer sequence of {n if n is not None else 'at least two'} entries")
    if a.size and (a.min() < 0 or a.max() >= 1 << 31):
        raise ValueError(f"{name} must lie in [0, 2^31)")
    return np.ascontiguousarray(a, dtype=np.int32)


def _sequences(graph_offsets, key_offsets, key_lengths):
    """Host arrays and their pointers, and the number of sequences."""
    qo = None if graph_offsets is None else _int32(graph_offsets, "graph_offsets")
    G = 1 if qo is None else len(qo) - 1
    ko = None if key_offsets is None else _int32(key_offsets, "key_offsets", G + 1)
    if qo is None and ko is not None:
        raise ValueError("key_offsets needs graph_offsets")
    kl = None if key_lengths is None else _int32(key_lengths, "key_lengths", G)
    arrays = (qo, ko, kl)
    return arrays, [ctypes.c_void_p(0 if a is None else a.ctypes.data) for a in arrays], G


def _sizes(q, k_, v):
    for t, name in ((q, "Q"), (k_, "K"), (v, "V")):
        if not isinstance(t, torch.Tensor) or t.dim() != 3:
            raise ValueError(f"{name} must be a tensor [N, heads, width]")
    return q.shape[0], k_.shape[0], q.shape[1], k_.shape[1], q.shape[2], v.shape[2]


def _inputs(q, k_, v, *more):
    """Checks Q, K, V (and more (tensor, name, shape) of their type); returns sizes, strides (host int64) and dtype code."""
    Nq, Nk, H, Hk, d, dv = _sizes(q, k_, v)
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise TypeError(f"Q must be torch.bfloat16 or torch.float16, got {q.dtype}")
    strides = []
    for t, name, shape in ((q, "Q", (Nq, H, d)), (k_, "K", (Nk, Hk, d)), (v, "V", (Nk, Hk, dv)), *more):
        strides.extend(_check_view(t, name, q.dtype, shape))
    return (Nq, Nk, H, Hk, d, dv), (ctypes.c_int64 * len(strides))(*strides), _DTYPES[q.dtype]


def _output(t, name, dtype, shape, device):
    """t (checked) or a new tensor."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _check_view(t, name, dtype, shape)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _scratch(workspace, nbytes, device):
    if nbytes == 0:
        return None
    if workspace is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    buf = workspace.get(nbytes)
    if buf.device != device:
        raise ValueError(f"workspace is on {buf.device}, expected {device}")
    return buf


def full_fwd_workspace_size(Nq: int, Nk: int, H: int, Hk: int, d: int, dv: int, graph_offsets=None, key_offsets=None,
                            key_lengths=None) -> int:
    keep, ptrs, G = _sequences(graph_offsets, key_offsets, key_lengths)
    return int(load().kmip_full_fwd_workspace_size(*ptrs, G, Nq, Nk, H, Hk, d, dv))


def full_fwd(q, k_, v, scale: float, graph_offsets: Optional[Sequence[int]] = None, key_offsets=None, key_lengths=None,
             causal: bool = False, out=None, lse=None, workspace=None):
    """Full softmax attention: returns (out, lse)."""
    (Nq, Nk, H, Hk, d, dv), strides, code = _inputs(q, k_, v)
    given = [(t, n) for t, n in ((out, "out"), (lse, "lse")) if t is not None]
    if out is not None:
        _output(out, "out", q.dtype, (Nq, H, dv), None)
    if lse is not None:
        _output(lse, "lse", torch.float32, (Nq, H), None)
    keep, ptrs, G = _sequences(graph_offsets, key_offsets, key_lengths)
    dev = _check_devices((q, "Q"), (k_, "K"), (v, "V"), *given)
    out = _output(out, "out", q.dtype, (Nq, H, dv), dev)
    lse = _output(lse, "lse", torch.float32, (Nq, H), dev)
    lib = load()
    buf = _scratch(workspace, lib.kmip_full_fwd_workspace_size(*ptrs, G, Nq, Nk, H, Hk, d, dv), dev)
    with _on_device(dev) as stream:
        check(lib.kmip_full_fwd(_ptr(q), _ptr(k_), _ptr(v), code, strides, *ptrs, G, Nq, Nk, H, Hk, d, dv, float(scale),
                                int(bool(causal)), _ptr(out), _ptr(lse), _ptr(buf), 0 if buf is None else buf.numel(),
                                stream))
    return out, lse


def full_bwd_workspace_size(Nq: int, Nk: int, H: int, Hk: int, d: int, dv: int, graph_offsets=None, key_offsets=None,
                            key_lengths=None) -> int:
    keep, ptrs, G = _sequences(graph_offsets, key_offsets, key_lengths)
    return int(load().kmip_full_bwd_workspace_size(*ptrs, G, Nq, Nk, H, Hk, d, dv))


def full_bwd(q, k_, v, dout, out, lse, scale: float, graph_offsets: Optional[Sequence[int]] = None, key_offsets=None,
             key_lengths=None, causal: bool = False, dq=None, dk=None, dv=None, workspace=None):
    """Gradients of full softmax attention: returns (dQ, dK, dV) of the inputs' type."""
    Nq, Nk, H, Hk, d, wv = _sizes(q, k_, v)
    sizes, strides, code = _inputs(q, k_, v, (dout, "dOut", (Nq, H, wv)))
    _output(out, "out", q.dtype, (Nq, H, wv), None)
    _output(lse, "lse", torch.float32, (Nq, H), None)
    shapes = ((dq, "dQ", (Nq, H, d)), (dk, "dK", (Nk, Hk, d)), (dv, "dV", (Nk, Hk, wv)))
    given = [(t, n) for t, n, shape in shapes if t is not None and _output(t, n, q.dtype, shape, None) is not None]
    keep, ptrs, G = _sequences(graph_offsets, key_offsets, key_lengths)
    dev = _check_devices((q, "Q"), (k_, "K"), (v, "V"), (dout, "dOut"), (out, "out"), (lse, "lse"), *given)
    dq, dk, dv = (_output(t, n, q.dtype, shape, dev) for t, n, shape in shapes)
    lib = load()
    buf = _scratch(workspace, lib.kmip_full_bwd_workspace_size(*ptrs, G, *sizes), dev)
    with _on_device(dev) as stream:
        check(lib.kmip_full_bwd(_ptr(q), _ptr(k_), _ptr(v), _ptr(dout), _ptr(out), _ptr(lse), code, strides, *ptrs, G,
                                *sizes, float(scale), int(bool(causal)), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(buf),
                                0 if buf is None else buf.numel(), stream))
    return dq, dk, dv


def full_attention(q, k_, v, scale: float, graph_offsets: Optional[Sequence[int]] = None, key_offsets=None,
                   key_lengths=None, causal: bool = False, workspace=None):
    """Differentiable full softmax attention: returns out [Nq, H, dv] of the inputs' type.

    The forward is ``full_fwd``; autograd's backward calls ``full_bwd`` with
    the saved out and lse.  Once differentiable.
    """
    where = dict(graph_offsets=graph_offsets, key_offsets=key_offsets, key_lengths=key_lengths, causal=causal)
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
            if dout.stride(-1) != 1 or any(s % 8 for s in dout.stride()[:2]) or dout.data_ptr() % 16:
                dout = dout.contiguous()
            return (*full_bwd(q, k_, v, dout, out, lse, scale, workspace=workspace, **where), None, None, None)

    return _Full
