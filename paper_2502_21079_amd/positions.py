"""Rotary positions of queries and keys, as a video transformer's own attention
takes them (by frame, row and column) and a text decoder's (by place).

Argument marshalling only, as in the package's other calls: every step runs in
the HIP kernel of ``libadaspa.so`` (the C ABI is in ``include/adaspa.h``).

* :func:`rotary`, :func:`rotary_bwd`    queries and keys turned by their positions
      in one call, and the gradients turned back
* :func:`rotary_embedding`              the same as a function that autograd
      differentiates
* :func:`rotary_frequencies`, :func:`rotary_magnitude`    the angle per position of
      each pair, also scaled for contexts longer than trained

Tensors are bf16 or fp16 views [B, heads, tokens, D] with D contiguous (a
multiple of 8, up to 256); other strides are the caller's, multiples of 8.
"""
from __future__ import annotations

import ctypes
import functools
import math
from operator import index
from typing import Optional, Sequence, Union

import torch
from torch.autograd.function import once_differentiable

from . import AdaspaError, _check, _on, _ptr, _stream, load_library
from .prompt import _DTYPES, _I64x3, _new, _new_strides, _steps

__all__ = ["rotary", "rotary_bwd", "rotary_embedding", "rotary_frequencies", "rotary_magnitude"]

_LAYOUTS = {"half": 0, "interleaved": 1}
_FLOATS = {float}


class _RotaryProblem(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("batch", "heads", "kv_heads", "len", "head_dim", "dtype", "pairs",
                                               "layout", "axes")]
                + [("axis_pairs", ctypes.c_int32 * 4), ("magnitude", ctypes.c_float),
                   ("freq", ctypes.POINTER(ctypes.c_double))]
                + [(n + "_stride", _I64x3) for n in ("q", "k", "q_out", "k_out")]
                + [("position_stride", ctypes.c_int64 * 2)])


# --- frequencies ---------------------------------------------------------------

def rotary_frequencies(dims: int, base: float = 10000.0, *, sections: Optional[Sequence[int]] = None,
                       scaling: Optional[str] = None, factor: float = 1.0, context: int = 0, low: float = 1.0,
                       high: float = 32.0):
    """Radians per position of each pair of the first ``dims`` elements of a
    head, as a tuple: base^(-2 i / d) for pair i of the d elements of an axis.

    ``sections`` gives the pairs of each axis (frame, row, column), one after
    another and dims / 2 in all; None is one axis.  For contexts ``factor``
    times longer than trained, ``scaling`` is

    * "linear": every frequency divided by factor (positions interpolated);
    * "base": the base times factor^(d / (d - 2)), which leaves the fastest pair
      as it is and divides the slowest by factor;
    * "parts": pairs that turn at least ``high`` times over the ``context``
      trained positions stay, those that turn at most ``low`` times are divided
      by factor, those between blend linearly in their number of turns ("NTK by
      parts", arXiv 2309.00071, whose factor on the turned values is
      :func:`rotary_magnitude`)."""
    dims, factor = index(dims), float(factor)
    sections = (dims // 2,) if sections is None else tuple(map(index, sections))
    if dims < 2 or dims % 2 or sum(sections) != dims // 2 or min(sections) < 0:
        raise AdaspaError(f"dims must be even and the sections' pairs add up to its half, got {dims} and {sections}")
    if scaling not in (None, "linear", "base", "parts"):
        raise AdaspaError(f"unknown scaling {scaling!r}")
    if not base > 0 or not math.isfinite(base) or not factor > 0 or not math.isfinite(factor):
        raise AdaspaError(f"base and factor must be above 0 and finite, got {base} and {factor}")
    if scaling == "parts" and (index(context) < 1 or not low < high):
        raise AdaspaError(f"scaling by parts needs the trained context and low < high, got {context}, {low}, {high}")
    freqs = []
    for n in sections:
        d = 2 * n
        b = base * factor ** (d / (d - 2)) if scaling == "base" and d > 2 else base
        for i in range(n):
            f = float(b) ** (-2 * i / d)
            if scaling == "linear":
                f /= factor
            elif scaling == "parts":
                stay = min(1.0, max(0.0, (context * f / (2 * math.pi) - low) / (high - low)))
                f = f * stay + f / factor * (1 - stay)
            freqs.append(f)
    return tuple(freqs)


def rotary_magnitude(factor: float) -> float:
    """0.1 ln(factor) + 1 (1 up to a factor of 1): the factor on the turned
    queries and keys that goes with "parts"."""
    return 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0


# --- plans: argument structures, once per set of values --------------------------

class _Plan:
    __slots__ = ("prob", "struct")


@functools.lru_cache(maxsize=512, typed=True)
def _plan(dtype, shapes, strides, outs, freqs, layout, sections, magnitude, pos_shape, pos_stride) -> _Plan:
    """Checks the shapes and strides of q, k and the positions and the strides of
    the outputs (None: new ones of the inputs' layout) and sets up the call's
    structure."""
    qs, ks = shapes
    if len(qs) != 4 or (ks is not None and (len(ks) != 4 or ks[0] != qs[0] or ks[2:] != qs[2:])):
        raise AdaspaError(f"q and k must be [B, heads, tokens, D] and differ in heads alone, got {qs} and {ks}")
    if layout not in _LAYOUTS:
        raise AdaspaError(f"unknown layout {layout!r}: 'half' or 'interleaved'")
    sections = (len(freqs),) if sections is None else sections
    if not 1 <= len(sections) <= 4 or min(sections) < 0 or sum(sections) != len(freqs):
        raise AdaspaError(f"sections must be up to 4 numbers of pairs that add up to {len(freqs)}, got {sections}")
    if not 1 <= len(freqs) <= qs[3] // 2:
        raise AdaspaError(f"freqs must have one entry per turned pair, 1 to D / 2 = {qs[3] // 2}, got {len(freqs)}")
    if max(*qs, *(ks or ())) >= 1 << 31:              # the structure's numbers would wrap
        raise AdaspaError(f"sizes must be below 2^31, got q {qs} and k {ks}")
    B, H, L, D = qs
    p = _RotaryProblem(B, H, 0 if ks is None else ks[1], L, D, dtype, len(freqs), _LAYOUTS[layout], len(sections),
                       (ctypes.c_int32 * 4)(*sections), magnitude)
    arr = (ctypes.c_double * len(freqs))(*freqs)
    p.freq = ctypes.cast(arr, ctypes.POINTER(ctypes.c_double))
    for name, n, s, o in zip(("q", "k"), shapes, strides, outs):
        if n is not None:
            setattr(p, name + "_stride", _I64x3(*_steps(n, s)))
            setattr(p, name + "_out_stride", _I64x3(*_steps(n, _new_strides(n, s) if o is None else o)))
    if pos_shape is not None:
        axes = () if len(sections) == 1 else (len(sections),)
        if pos_shape == (L,) + axes:
            step = (0, pos_stride[0] if L > 1 else 0)
        elif pos_shape in ((B, L) + axes, (1, L) + axes):
            step = (pos_stride[0] if pos_shape[0] > 1 else 0, pos_stride[1] if L > 1 else 0)
        else:
            raise AdaspaError(f"positions must be [tokens] or [B, tokens]{', the axes last' if axes else ''}: "
                              f"{(B, L) + axes}, got {pos_shape}")
        if axes and pos_stride[-1] != 1:
            raise AdaspaError("the axes of a position must be contiguous")
        p.position_stride = (ctypes.c_int64 * 2)(*step)
    elif len(sections) > 1:
        raise AdaspaError("several axes need positions")
    p._arr = arr                                      # lives as long as the structure that points to it
    plan = _Plan()
    plan.struct, plan.prob = p, ctypes.byref(p)
    return plan


def _check_int32(t, name, dev):
    if t.dtype is not torch.int32 or t.get_device() != dev:
        raise AdaspaError(f"{name} must be an int32 tensor on q's device")


def _turn(call, q, k, freqs, layout, sections, magnitude, positions, offset, out, k_out):
    dev = q.get_device()
    if dev < 0 or q.dtype not in _DTYPES:
        raise AdaspaError("q and k must be bf16 or fp16 CUDA tensors [B, heads, tokens, D]")
    if k is not None and (k.dtype is not q.dtype or k.get_device() != dev):
        raise AdaspaError("q and k must share one type and device")
    for o, x, name in ((out, q, "out"), (k_out, k, "k_out")):
        if o is not None and (x is None or o.dtype is not x.dtype or o.shape != x.shape or o.device != x.device):
            raise AdaspaError(f"{name} must be a tensor of its input's type and shape on its device")
    if positions is not None:
        _check_int32(positions, "positions", dev)
    offsets = None
    if isinstance(offset, torch.Tensor):
        offset, offsets = 0, offset
        _check_int32(offsets, "offset", dev)
        if offsets.shape != q.shape[:1] or not offsets.is_contiguous():
            raise AdaspaError(f"offset must be a number or a contiguous int32 [B] = {tuple(q.shape[:1])} tensor")
    else:
        offset = index(offset)
        if not -(1 << 40) < offset < 1 << 40:
            raise AdaspaError(f"offset must be below 2^40 in magnitude, got {offset}")
    if type(freqs) is not tuple or set(map(type, freqs)) != _FLOATS:
        freqs = tuple(map(float, freqs))              # plain numbers: a plan is kept by them
    plan = _plan(_DTYPES[q.dtype], (q.shape, None if k is None else k.shape),
                 (q.stride(), None if k is None else k.stride()),
                 (None if out is None else out.stride(), None if k_out is None else k_out.stride()),
                 freqs, layout, None if sections is None else tuple(map(index, sections)), float(magnitude),
                 None if positions is None else positions.shape, None if positions is None else positions.stride())
    out = _new(q) if out is None else out
    if k is not None and k_out is None:
        k_out = _new(k)
    with _on(dev):
        _check(call(plan.prob, q.data_ptr(), _ptr(k), _ptr(positions), offset, _ptr(offsets), out.data_ptr(),
                    _ptr(k_out), _stream(q.device)))
    return out, k_out


# --- calls -----------------------------------------------------------------------

def rotary(q, k, freqs, *, layout: str = "half", sections=None, magnitude: float = 1.0, positions=None,
           offset: Union[int, torch.Tensor] = 0, out=None, k_out=None):
    """q [B, H, L, D] and k [B, Hk, L, D] (or None) turned by their positions.
    Returns (out, k_out).

    Pair i of a head is turned by its token's position times ``freqs[i]`` (a tuple
    of radians, :func:`rotary_frequencies`) and multiplied by ``magnitude``; what
    lies behind the pairs is copied.  Pairs are elements (i, i + n) of the n pairs
    (``layout`` "half") or (2 i, 2 i + 1) ("interleaved").  The position is that of
    ``positions`` (int32 [L] or [B, L]; None: the token's place) plus ``offset`` (a
    number, or int32 [B]: the tokens that a cache holds already).  With several
    ``sections`` (pairs of each axis, in order) a position has a number per axis,
    int32 [L, axes] or [B, L, axes].  Angles are formed in 64 bits.

    ``out`` and ``k_out`` may be q and k themselves; other tensors must not overlap
    them."""
    return _turn(load_library().adaspa_rotary, q, k, freqs, layout, sections, magnitude, positions, offset, out, k_out)


def rotary_bwd(dout, dk_out, freqs, *, layout: str = "half", sections=None, magnitude: float = 1.0, positions=None,
               offset: Union[int, torch.Tensor] = 0, dq=None, dk=None):
    """Gradients (dq, dk) of :func:`rotary` from those of its results (``dk_out``
    may be None); the other arguments are what it was given."""
    return _turn(load_library().adaspa_rotary_bwd, dout, dk_out, freqs, layout, sections, magnitude, positions, offset,
                 dq, dk)


# --- autograd ----------------------------------------------------------------------

def _rows(t):
    """t itself where the kernel can read it as it lies, else a copy."""
    try:
        _steps(t.shape, t.stride())
        readable = t.data_ptr() % 16 == 0
    except AdaspaError:
        readable = False
    return t if readable else t.clone(memory_format=torch.contiguous_format)


class _RotaryEmbedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, offset, freqs, kw):
        ctx.set_materialize_grads(False)
        ctx.freqs, ctx.kw = freqs, kw
        ctx.number = None if isinstance(offset, torch.Tensor) else offset
        ctx.save_for_backward(positions, None if ctx.number is not None else offset)
        return rotary(q, k, freqs, positions=positions, offset=offset, **kw)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, dk_out):
        positions, offset = ctx.saved_tensors
        kw = dict(ctx.kw, positions=positions, offset=offset if ctx.number is None else ctx.number)
        dout = _rows(dout) if dout is not None and ctx.needs_input_grad[0] else None
        dk_out = _rows(dk_out) if dk_out is not None and ctx.needs_input_grad[1] else None
        if dout is None:
            dk = None if dk_out is None else rotary_bwd(dk_out, None, ctx.freqs, **kw)[0]
            return None, dk, None, None, None, None
        return (*rotary_bwd(dout, dk_out, ctx.freqs, **kw), None, None, None, None)


def rotary_embedding(q, k, freqs, *, layout: str = "half", sections=None, magnitude: float = 1.0, positions=None,
                     offset: Union[int, torch.Tensor] = 0):
    """What :func:`rotary` returns, differentiable (once) in q and k.  A backward pass may be
    captured into a graph with its forward pass; as with any function of torch's, no graph of
    the same leaves from outside the capture may be alive then."""
    kw = dict(layout=layout, sections=sections, magnitude=magnitude)
    return _RotaryEmbedding.apply(q, k, positions, offset, tuple(map(float, freqs)), kw)


def _declare(lib):
    """Argument types of the library's calls."""
    P, vp = ctypes.POINTER(_RotaryProblem), ctypes.c_void_p
    for name in ("adaspa_rotary", "adaspa_rotary_bwd"):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = ctypes.c_int, [P, vp, vp, vp, ctypes.c_int64, vp, vp, vp, vp]
