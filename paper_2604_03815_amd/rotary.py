"""Rotary positions on queries and keys: front end of kmip_rotary.

Pair i of a row's first ``rot = 2 len(freqs)`` dimensions (neighbours 2i, 2i + 1
where ``interleaved``, else dimensions i and i + rot / 2) is turned by
position * freqs[i] radians and scaled by ``magnitude``; the rest of the row is
passed on.  The scores of turned queries and keys depend on the difference of their positions.
"""
from __future__ import annotations

import functools
import math
from typing import Optional

import numpy as np
import torch
from torch.autograd import forward_ad

from ._lib import load
from .full import _DTYPES, _address, _check_devices, _check_tensor, _check_written, _launch as _launch_on, _new, _strides, _written


def rotary_frequencies(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                       original_length: Optional[int] = None, slow_turns: float = 1.0, fast_turns: float = 32.0):
    """(freqs float64 [rot / 2] in radians a position, magnitude) for ``rotary``.

    freqs[i] = base^(-2 i / rot); for contexts ``factor`` times longer than the ``original_length`` trained on:
      "linear"  every frequency divided by the factor;
      "base"    base times factor^(rot / (rot - 2)): the fastest pair as it was, the slowest divided by the factor;
      "blend"   pairs that turn less than ``slow_turns`` times in the original length divided by the factor, those that turn more
                than ``fast_turns`` times as they were, a linear blend in between; magnitude 0.1 log(factor) + 1 (1 for a factor below 1).
    """
    if rot < 2 or rot % 2:
        raise ValueError("rot must be even and at least 2")
    if not base > 0 or not factor > 0:
        raise ValueError("base and factor must be > 0")
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    freqs = base ** (-2.0 * np.arange(rot // 2, dtype=np.float64) / rot)
    if scaling in ("none", "base"):
        return freqs, 1.0
    if scaling == "linear":
        return freqs / factor, 1.0
    if scaling != "blend":
        raise ValueError('scaling must be "none", "linear", "base" or "blend"')
    if original_length is None or not 0 <= slow_turns < fast_turns:
        raise ValueError("blend needs original_length and 0 <= slow_turns < fast_turns")
    keep = np.clip((original_length * freqs / (2 * math.pi) - slow_turns) / (fast_turns - slow_turns), 0.0, 1.0)
    return freqs * keep + freqs / factor * (1.0 - keep), 0.1 * math.log(max(factor, 1.0)) + 1.0


class Rotary:
    """Frequencies and layout of rotary positions, for the layers: a call turns q and k (see ``rotary``).

    rot: dimensions turned; the other arguments as in ``rotary_frequencies``.
    """

    def __init__(self, rot: int, interleaved: bool = False, **scaling):
        self.freqs, self.magnitude = rotary_frequencies(rot, **scaling)
        self.rot, self.interleaved = rot, interleaved

    def __call__(self, q, k_=None, positions=None, dtype=None):
        return rotary(q, k_, positions, self.freqs, interleaved=self.interleaved, magnitude=self.magnitude, dtype=dtype)


def _rows(t, name):
    if not isinstance(t, torch.Tensor) or t.dim() != 3:
        raise ValueError(f"{name} must be a tensor [N, heads, d]")
    if t.dtype not in _DTYPES:
        raise TypeError(f"{name} must be bfloat16, float16 or float32, got {t.dtype}")


def rotary(q, k_=None, positions=None, freqs=None, interleaved: bool = False, magnitude: float = 1.0, inverse: bool = False,
           dtype=None, q_out=None, k_out=None):
    """Turns q [N, H, d], and k_ [N, Hk, d] if given, to their positions in one launch: returns q, or (q, k).

    positions: int32 [N] on the device (None: row i is at position i); freqs: host float64 [rot / 2] (``rotary_frequencies``); dtype of the results
    (default: the inputs'): bfloat16, float16 or float32.  inverse turns back.  q_out, k_out: tensors to write into,
    q_out=q for in place.  Inputs and outputs may be views whose last dimension is contiguous (outputs must not overlap themselves).
    Differentiable in q and k_ unless q_out or k_out is given; once, and in reverse mode only (dual tensors are refused).
    For a backward in a HIP graph see ``full_attention``.
    """
    if freqs is None:
        raise ValueError("freqs must be given (see rotary_frequencies)")
    given = q_out is not None or k_out is not None
    grad = torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad for t in (q, k_))
    if grad or forward_ad._current_level >= 0 and _has_tangent(q, k_):
        # (dual tensors go this way too: autograd refuses them, the launch would drop their tangents)
        if given:
            raise ValueError("q_out and k_out are not differentiable: leave them out, or call under torch.no_grad()")
        _rows(q, "q")
        if k_ is not None and not isinstance(k_, torch.Tensor):
            raise ValueError("k must be a tensor [N, heads, d]")
        got = _rotary_function().apply(q, k_, positions, freqs, interleaved, magnitude, inverse, dtype)
        return got[0] if k_ is None else got
    return _launch(q, k_, positions, freqs, interleaved, magnitude, inverse, dtype, q_out, k_out)


def _has_tangent(*tensors):
    return any(isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None for t in tensors)


def _launch(q, k_, positions, freqs, interleaved, magnitude, inverse, dtype, q_out, k_out):
    _rows(q, "q")
    f = np.ascontiguousarray(freqs, dtype=np.float64)
    if f.ndim != 1:
        raise ValueError("freqs must be 1-D")
    N, H, d = q.shape
    H2, whole = 0, True
    if k_ is not None:
        _rows(k_, "k")
        H2 = k_.shape[1]
        whole = _check_tensor(k_, "k", q.dtype, (N, H2, d))
    elif k_out is not None:
        raise ValueError("k_out without k")
    to = q.dtype if dtype is None else dtype
    if to not in _DTYPES:
        raise TypeError(f"dtype must be bfloat16, float16 or float32, got {to}")
    whole &= _check_tensor(q, "q", q.dtype, (N, H, d))
    whole &= _check_out(q_out, "q_out", to, (N, H, d))
    whole &= _check_out(k_out, "k_out", to, (N, H2, d))
    if positions is not None:
        _check_positions(positions, N)
    dev = _check_devices((q, "q"), (k_, "k"), (q_out, "q_out"), (k_out, "k_out"), (positions, "positions"))
    given = q_out, k_out
    if q_out is None:
        q_out = _new(q, (N, H, d), to)
    if k_ is not None and k_out is None:
        k_out = _new(k_, (N, H2, d), to)
    strides = None
    if not whole:
        strides = _strides(q, q_out) if k_ is None else _strides(q, q_out, k_, k_out)
    _launch_on(dev, load().kmip_rotary, q.data_ptr(), q_out.data_ptr(), H, _address(k_), _address(k_out), H2, _DTYPES[q.dtype],
               _DTYPES[to], strides, _address(positions), f.__array_interface__["data"][0], N, d, 2 * len(f), 1 if interleaved else 0,
               float(magnitude), 1 if inverse else 0)
    _written(*given)
    return q_out if k_ is None else (q_out, k_out)


def _check_out(t, name, dtype, shape):
    if t is None:
        return True
    whole = _check_tensor(t, name, dtype, shape)
    _check_written(t, name)
    if whole:
        return True
    N, heads, d = shape
    if t.numel():
        rows, cols = (t.stride(0), N), (t.stride(1), heads)
        # one of the two dimensions within the other's steps, rows of d values within the smaller's
        inner, outer = sorted(x for x in (rows, cols) if x[1] > 1) if N > 1 and heads > 1 else ((d, 1), max(rows, cols, key=lambda x: x[1]))
        if inner[0] < d or (outer[1] > 1 and outer[0] < (inner[1] - 1) * inner[0] + d):
            raise ValueError(f"{name} overlaps itself")
    return False


def _check_positions(positions, N):
    if not isinstance(positions, torch.Tensor):
        raise TypeError("positions must be a torch tensor")
    if positions.dtype != torch.int32:
        raise TypeError(f"positions must be torch.int32, got {positions.dtype}")
    if tuple(positions.shape) != (N,):
        raise ValueError(f"positions must have shape {(N,)}, got {tuple(positions.shape)}")
    if not positions.is_contiguous():
        raise ValueError("positions must be contiguous")


@functools.lru_cache(maxsize=None)
def _rotary_function():
    class _Rotary(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k_, positions, freqs, interleaved, magnitude, inverse, dtype):
            freqs = np.array(freqs, dtype=np.float64)   # (the caller may change its own)
            got = _launch(q, k_, positions, freqs, interleaved, magnitude, inverse, dtype, None, None)
            ctx.save_for_backward(*(() if positions is None else (positions,)))
            ctx.args = freqs, interleaved, magnitude, inverse, q.dtype, k_ is not None
            return (got,) if k_ is None else got

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dq, dk=None):
            freqs, interleaved, magnitude, inverse, dtype, both = ctx.args
            positions = ctx.saved_tensors[0] if ctx.saved_tensors else None
            dq, dk = (t if t is None or t.shape[-1] < 2 or t.stride(-1) == 1 else t.contiguous() for t in (dq, dk))
            got = _launch(dq, dk, positions, freqs, interleaved, magnitude, not inverse, dtype, None, None)
            return (*(got if both else (got, None)), None, None, None, None, None, None)

    return _Rotary
