"""The prompt side of a video diffusion transformer: cross attention to a text
encoder's states, and the encoder's own attention with a learned relative
position bias.

Argument marshalling only, as in the package's other calls: every step runs in
the HIP kernels of ``libadaspa.so`` (the C ABI is in ``include/adaspa.h``).

* :func:`cross_attn`, :func:`cross_attn_bwd`        queries of one length over
      keys and values of another, with per-sample key lengths and key masks
* :func:`rel_bias_attn`, :func:`rel_bias_attn_bwd`  the same with a learned
      value per head and bucket of the distance added to the scores
* :func:`cross_attention`, :func:`rel_bias_attention`  the two as functions
      that autograd differentiates
* :func:`relative_bucket_starts`                    the buckets' first distances

Tensors are bf16 or fp16 views [B, heads, tokens, D] with D contiguous; other
strides are the caller's (a projection's [B, tokens, heads, D] output is passed
as its transpose).  ``scale`` multiplies the scores; None, and every value that is not
above 0 in fp32, stands for 1 / sqrt(D).
"""
from __future__ import annotations

import ctypes
import functools
from operator import index
from typing import Optional, Union

import torch
from torch.autograd.function import once_differentiable

from . import AdaspaError, _check, _ptr, _stream, load_library

__all__ = ["cross_attn", "cross_attn_workspace", "cross_attn_bwd", "cross_attn_bwd_workspace", "cross_attention",
           "rel_bias_attn", "rel_bias_attn_workspace", "rel_bias_attn_bwd", "rel_bias_attn_bwd_workspace",
           "rel_bias_attention", "relative_bucket_starts"]

_DTYPES = {torch.bfloat16: 0, torch.float16: 1}
_I64x3 = ctypes.c_int64 * 3
_NO_OUTPUTS = (None,) * 4
_NO_WORKSPACE = 16                        # the size of a call that takes none


class _CrossProblem(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("batch", "heads", "kv_heads", "q_len", "k_len", "head_dim", "dtype")]
                + [("softmax_scale", ctypes.c_float)]
                + [(n + "_stride", _I64x3) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")]
                + [("key_mask_stride", ctypes.c_int64)])


class _RelBias(ctypes.Structure):
    _fields_ = [("num_buckets", ctypes.c_int32), ("bidirectional", ctypes.c_int32),
                ("bucket_start", ctypes.POINTER(ctypes.c_int32)), ("causal", ctypes.c_int32),
                ("q_offset", ctypes.c_int32), ("queries_at_end", ctypes.c_int32), ("table_fp32", ctypes.c_int32)]


# --- plans: argument structures and sizes, once per set of values -------------

@functools.lru_cache(maxsize=256, typed=True)
def relative_bucket_starts(num_buckets: int, max_distance: int, bidirectional: bool = True):
    """First distance of each bucket of one direction, as a tuple.

    A direction has n = ``num_buckets`` buckets, half of them when
    ``bidirectional``.  The first e = n // 2 hold one distance each; from e on
    they widen logarithmically, bucket e + m beginning at the least distance d
    with (d / e)^(n - e) >= (max_distance / e)^m, compared in whole numbers."""
    num_buckets, max_distance = index(num_buckets), index(max_distance)
    n = num_buckets // 2 if bidirectional else num_buckets
    if n < 2 or (bidirectional and num_buckets % 2):
        raise AdaspaError("num_buckets must be at least 2, or an even number of at least 4 when bidirectional")
    e = n // 2
    if max_distance <= e:
        raise AdaspaError(f"max_distance must be more than {e}, the distances with a bucket of their own")
    starts = list(range(e)) + [e]
    for m in range(1, n - e):
        low, high = starts[-1], max_distance          # the condition holds at max_distance
        while low < high:
            d = (low + high) // 2
            if d ** (n - e) * e ** m < max_distance ** m * e ** (n - e):
                low = d + 1
            else:
                high = d
        starts.append(low)
    return tuple(starts)


@functools.lru_cache(maxsize=512, typed=True)
def _bias_ref(num_buckets, max_distance, bidirectional, causal, q_offset, table_fp32):
    starts = relative_bucket_starts(num_buckets, max_distance, bidirectional)
    arr = (ctypes.c_int32 * len(starts))(*(min(d, (1 << 31) - 1) for d in starts))
    end = q_offset == "end"
    if not end and not -(1 << 28) < q_offset < 1 << 28:
        raise AdaspaError(f"q_offset must be below 2^28 in magnitude, got {q_offset}")
    r = _RelBias(num_buckets, int(bidirectional), ctypes.cast(arr, ctypes.POINTER(ctypes.c_int32)), int(causal),
                 0 if end else q_offset, int(end), int(table_fp32))
    r._starts = arr                       # lives as long as the structure that points to it
    return ctypes.byref(r)


class _Plan:
    """What calls on tensors of one set of shapes and strides share."""
    __slots__ = ("prob", "bias", "need", "rows")


@functools.lru_cache(maxsize=512)
def _plan(bwd, dtype, shapes, strides, outs, scale, mask_stride, bias) -> _Plan:
    """Checks the shapes and strides of q, k, v (and dout) and the strides of
    the outputs (None: new ones of the inputs' layout) and sets up the call's
    structures and workspace size."""
    lib = load_library()
    qs, ks, vs = shapes[:3]
    if len(qs) != 4 or len(ks) != 4:
        raise AdaspaError(f"q, k, v must be [B, heads, tokens, D], got {tuple(qs)} and {tuple(ks)}")
    if vs != ks or ks[0] != qs[0] or ks[3] != qs[3] or ks[1] == 0 or qs[1] % ks[1]:
        raise AdaspaError(f"shapes do not fit: q {tuple(qs)}, k {tuple(ks)}, v {tuple(vs)}")
    ins = [_steps(s, t) for s, t in zip(shapes, strides)]
    # Results in the order out, dq, dk, dv.
    like = ((qs, strides[0]), (qs, strides[0]), (ks, strides[1]), (ks, strides[2]))
    res = [_steps(n, _new_strides(n, t) if o is None else o) for (n, t), o in zip(like, outs)]
    B, H, Lq, D = qs
    if max(*qs, *ks) >= 1 << 31:                 # the structure's numbers would wrap
        raise AdaspaError(f"sizes must be below 2^31, got q {tuple(qs)} and k {tuple(ks)}")
    p = _CrossProblem(B, H, ks[1], Lq, ks[2], D, dtype, scale)
    for name, s in zip(("q", "k", "v", "dout", "out", "dq", "dk", "dv"), ins + [ins[0]] * (4 - len(ins)) + res):
        setattr(p, name + "_stride", _I64x3(*s))
    p.key_mask_stride = mask_stride
    plan = _Plan()
    plan.prob, plan.rows = ctypes.byref(p), (B, H, Lq)
    plan.bias = None if bias is None else _bias_ref(*bias)
    name = "adaspa_%s_attn%s_workspace" % ("cross" if bias is None else "rel_bias", "_bwd" if bwd else "")
    plan.need = int(getattr(lib, name)(plan.prob, *([] if bias is None else [plan.bias])))
    return plan


def _steps(shape, stride):
    """(batch, head, token) strides of a tensor the kernels can read, 0 in
    place of those that nothing steps along."""
    s = tuple(a if n > 1 else 0 for a, n in zip(stride[:3], shape))
    if stride[3] != 1 and shape[3] > 1 or (s[0] | s[1] | s[2]) & 7:
        raise AdaspaError("tensors need D contiguous and (batch, head, token) strides that are multiples of 8, got "
                          f"strides {tuple(stride)}")
    return s


@functools.lru_cache(maxsize=512)
def _keeps_layout(shape, stride):
    """Whether a new tensor like one of this shape gets these strides: no two
    elements in one place and no gaps."""
    n = 1
    for a, m in sorted((a, m) for a, m in zip(stride, shape) if m > 1):
        if a != n:
            return False
        n *= m
    return 0 not in shape


def _new_strides(shape, stride):
    return stride if _keeps_layout(shape, stride) else _contiguous(shape)


def _new(t):
    """A new tensor of t's shape, in its layout where that is kept."""
    return torch.empty_like(t) if _keeps_layout(t.shape, t.stride()) else \
        torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _contiguous(shape):
    B, H, L, D = shape
    return (H * L * D, L * D, D, 1)


# --- argument checks -----------------------------------------------------------

def _check_tensors(q, k, v):
    """The device index of q, k, v, after checks of type and device."""
    dev = q.get_device()
    if dev < 0 or q.dtype not in _DTYPES:
        raise AdaspaError("q, k, v must be bf16 or fp16 CUDA tensors [B, heads, tokens, D]")
    if k.dtype is not q.dtype or v.dtype is not q.dtype or k.get_device() != dev or v.get_device() != dev:
        raise AdaspaError("q, k, v must share one type and device")
    return dev


def _check_like(t, like, name):
    """Strides of a tensor that the caller gives for a result, or with one."""
    if t.dtype is not like.dtype or t.shape != like.shape or t.device != like.device:
        raise AdaspaError(f"{name} must be a {like.dtype} tensor of shape {tuple(like.shape)} on q's device")
    return t.stride()


def _check_lse(lse, q):
    if lse.dtype is not torch.float32 or lse.shape != q.shape[:3] or not lse.is_contiguous() or lse.device != q.device:
        raise AdaspaError(f"lse must be a contiguous fp32 [B, H, Lq] = {tuple(q.shape[:3])} tensor on q's device")


def _check_keys(key_lens, key_mask, q, k, dev):
    """Bytes between the mask's rows, after checks of lengths and mask."""
    if key_lens is not None and (key_lens.dtype is not torch.int32 or key_lens.shape != q.shape[:1]
                                 or not key_lens.is_contiguous() or key_lens.get_device() != dev):
        raise AdaspaError(f"key_lens must be a contiguous int32 [B] = {tuple(q.shape[:1])} tensor on q's device")
    if key_mask is None:
        return 0
    if key_mask.dtype not in (torch.bool, torch.uint8) or key_mask.shape != q.shape[:1] + k.shape[2:3] \
            or key_mask.get_device() != dev or (key_mask.stride(1) != 1 and key_mask.shape[1] > 1):
        raise AdaspaError(f"key_mask must be a bool or uint8 [B, Lk] = {tuple(q.shape[:1] + k.shape[2:3])} tensor with "
                          "contiguous rows on q's device")
    return key_mask.stride(0)


def _bias_key(q, k, table, max_distance, bidirectional, causal, q_offset):
    if table.dim() != 2 or table.shape[1] != q.shape[1] or not table.is_contiguous() or table.device != q.device \
            or table.dtype not in (torch.float32, q.dtype):
        raise AdaspaError(f"table must be a contiguous [num_buckets, H = {q.shape[1]}] tensor, fp32 or of q's type, on "
                          "q's device")
    if q_offset != "end":
        q_offset = index(q_offset)
    return (table.shape[0], index(max_distance), bool(bidirectional), bool(causal), q_offset,
            table.dtype is torch.float32)


def _scratch(workspace, need, q):
    """(workspace, bytes): the caller's, checked, or a new one; None where a
    call needs none."""
    if workspace is not None:
        if workspace.device != q.device or not workspace.is_contiguous():
            raise AdaspaError("workspace must be a contiguous tensor on q's device")
        return workspace, workspace.numel() * workspace.element_size()
    if need <= _NO_WORKSPACE:
        return None, 0
    return torch.empty(need, dtype=torch.uint8, device=q.device), need


# --- forward -------------------------------------------------------------------

def _forward(q, k, v, table, bias, key_lens, key_mask, scale, out, lse, want_lse, workspace):
    dev = _check_tensors(q, k, v)
    mask_stride = 0
    if key_lens is not None or key_mask is not None:
        mask_stride = _check_keys(key_lens, key_mask, q, k, dev)
    given = _NO_OUTPUTS if out is None else (_check_like(out, q, "out"), None, None, None)
    plan = _plan(False, _DTYPES[q.dtype], (q.shape, k.shape, v.shape), (q.stride(), k.stride(), v.stride()), given,
                 0.0 if scale is None else float(scale), mask_stride, bias)
    if out is None:
        out = _new(q)
    if lse is not None:
        _check_lse(lse, q)
    elif want_lse:
        lse = q.new_empty(plan.rows, dtype=torch.float32)
    workspace, ws_bytes = _scratch(workspace, plan.need, q)
    lib = load_library()
    if bias is None:
        status = lib.adaspa_cross_attn(plan.prob, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(key_lens),
                                       _ptr(key_mask), out.data_ptr(), _ptr(lse), _ptr(workspace), ws_bytes,
                                       _stream(q.device))
    else:
        status = lib.adaspa_rel_bias_attn(plan.prob, plan.bias, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                          table.data_ptr(), _ptr(key_lens), _ptr(key_mask), out.data_ptr(), _ptr(lse),
                                          _ptr(workspace), ws_bytes, _stream(q.device))
    _check(status)
    return out, lse


def cross_attn(q, k, v, *, key_lens=None, key_mask=None, scale: Optional[float] = None, out=None, lse=None,
               want_lse: bool = True, workspace=None):
    """Attention of q [B, H, Lq, D] over k, v [B, Hk, Lk, D] (H % Hk == 0, runs
    of H / Hk query heads share a key head).  Returns (out, lse).

    ``key_lens`` (int32 [B]) leaves sample b its first key_lens[b] keys,
    ``key_mask`` (bool or uint8 [B, Lk], 0 = masked) takes single ones away.  A
    row that sees no key gives 0 and an lse of -inf; what masked keys hold
    takes no part.  ``scale`` defaults to 1 / sqrt(D), which values up to 0 stand for
    too.  ``workspace`` (at least :func:`cross_attn_workspace` bytes,
    any type) is allocated here when not given and needed: few query rows
    split their keys over workgroups."""
    return _forward(q, k, v, None, None, key_lens, key_mask, scale, out, lse, want_lse, workspace)


def rel_bias_attn(q, k, v, table, *, max_distance: int = 128, bidirectional: bool = True, causal: bool = False,
                  q_offset: Union[int, str] = 0, key_lens=None, key_mask=None, scale: Optional[float] = None,
                  out=None, lse=None, want_lse: bool = True, workspace=None):
    """:func:`cross_attn` with ``table[bucket, h]`` added to the scaled scores,
    the bucket being that of key position minus query position
    (:func:`relative_bucket_starts`): ``table`` is [num_buckets, H], fp32 or of
    q's type.  When ``bidirectional`` the second half of its rows is for keys
    after the query; otherwise those count as distance 0.  Values of minus
    infinity, or past -2.3e38, hide their keys.  ``causal`` masks keys after the
    query.  ``scale`` as there: 0 is not "no scores" but 1 / sqrt(D).  Query i stands at
    position i + ``q_offset`` among the keys; "end"
    puts a sample's queries at its last positions (decoding with a cache: one
    query over key_lens[b] keys).  Returns (out, lse)."""
    bias = _bias_key(q, k, table, max_distance, bidirectional, causal, q_offset)
    return _forward(q, k, v, table, bias, key_lens, key_mask, scale, out, lse, want_lse, workspace)


# --- backward ------------------------------------------------------------------

def _backward(dout, q, k, v, table, bias, out, lse, key_lens, key_mask, scale, dq, dk, dv, workspace):
    dev = _check_tensors(q, k, v)
    mask_stride = 0
    if key_lens is not None or key_mask is not None:
        mask_stride = _check_keys(key_lens, key_mask, q, k, dev)
    _check_lse(lse, q)
    g = _check_like(dout, q, "dout")
    given = (_check_like(out, q, "out"),) + tuple(
        None if x is None else _check_like(x, t, n) for x, t, n in ((dq, q, "dq"), (dk, k, "dk"), (dv, v, "dv")))
    plan = _plan(True, _DTYPES[q.dtype], (q.shape, k.shape, v.shape, q.shape), (q.stride(), k.stride(), v.stride(), g),
                 given, 0.0 if scale is None else float(scale), mask_stride, bias)
    dq = _new(q) if dq is None else dq
    dk = _new(k) if dk is None else dk
    dv = _new(v) if dv is None else dv
    workspace, ws_bytes = _scratch(workspace, plan.need, q)
    lib = load_library()
    if bias is None:
        _check(lib.adaspa_cross_attn_bwd(plan.prob, dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                         _ptr(key_lens), _ptr(key_mask), out.data_ptr(), lse.data_ptr(), dq.data_ptr(),
                                         dk.data_ptr(), dv.data_ptr(), _ptr(workspace), ws_bytes, _stream(q.device)))
        return dq, dk, dv
    dtable = torch.empty_like(table)
    _check(lib.adaspa_rel_bias_attn_bwd(plan.prob, plan.bias, dout.data_ptr(), q.data_ptr(), k.data_ptr(),
                                        v.data_ptr(), table.data_ptr(), _ptr(key_lens), _ptr(key_mask), out.data_ptr(),
                                        lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), dtable.data_ptr(),
                                        _ptr(workspace), ws_bytes, _stream(q.device)))
    return dq, dk, dv, dtable


def cross_attn_bwd(dout, q, k, v, out, lse, *, key_lens=None, key_mask=None, scale: Optional[float] = None,
                   dq=None, dk=None, dv=None, workspace=None):
    """Gradients (dq, dk, dv) of :func:`cross_attn` from the gradient of its
    output; ``out`` and ``lse`` are what it returned, the other arguments what
    it was given.  dk and dv are sums over the query heads that share a key
    head, and 0 for masked keys."""
    return _backward(dout, q, k, v, None, None, out, lse, key_lens, key_mask, scale, dq, dk, dv, workspace)


def rel_bias_attn_bwd(dout, q, k, v, table, out, lse, *, max_distance: int = 128, bidirectional: bool = True,
                      causal: bool = False, q_offset: Union[int, str] = 0, key_lens=None, key_mask=None,
                      scale: Optional[float] = None, dq=None, dk=None, dv=None, workspace=None):
    """Gradients (dq, dk, dv, dtable) of :func:`rel_bias_attn`; dtable, of the
    table's shape and type, is the sum over samples and over the pairs of each
    bucket."""
    bias = _bias_key(q, k, table, max_distance, bidirectional, causal, q_offset)
    return _backward(dout, q, k, v, table, bias, out, lse, key_lens, key_mask, scale, dq, dk, dv, workspace)


# --- workspaces ----------------------------------------------------------------

def _workspace(bwd, q_shape, k_shape, bias):
    qs, ks = tuple(map(index, q_shape)), tuple(map(index, k_shape))
    a, c = _contiguous(qs), _contiguous(ks)
    return _plan(bwd, 0, (qs, ks, ks), (a, c, c), _NO_OUTPUTS, 0.0, 0, bias).need


def cross_attn_workspace(q_shape, k_shape) -> int:
    """Bytes of the workspace of :func:`cross_attn` for q and k of these shapes."""
    return _workspace(False, q_shape, k_shape, None)


def cross_attn_bwd_workspace(q_shape, k_shape) -> int:
    """Bytes of the workspace of :func:`cross_attn_bwd`."""
    return _workspace(True, q_shape, k_shape, None)


def rel_bias_attn_workspace(q_shape, k_shape, num_buckets: int, *, max_distance: int = 128,
                            bidirectional: bool = True, causal: bool = False) -> int:
    """Bytes of the workspace of :func:`rel_bias_attn`."""
    return _workspace(False, q_shape, k_shape, (index(num_buckets), index(max_distance), bool(bidirectional), bool(causal),
                                                0, False))


def rel_bias_attn_bwd_workspace(q_shape, k_shape, num_buckets: int, *, max_distance: int = 128,
                                bidirectional: bool = True, causal: bool = False) -> int:
    """Bytes of the workspace of :func:`rel_bias_attn_bwd`."""
    return _workspace(True, q_shape, k_shape, (index(num_buckets), index(max_distance), bool(bidirectional), bool(causal),
                                                0, False))


# --- autograd ------------------------------------------------------------------

def _rows(t):
    """t itself where the kernels can read it as it lies, else a copy."""
    try:
        readable = _steps(t.shape, t.stride())[2] < 1 << 23 and t.data_ptr() % 16 == 0
    except AdaspaError:
        readable = False
    return t if readable else t.clone(memory_format=torch.contiguous_format)


class _CrossAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, key_lens, key_mask, scale):
        out, lse = cross_attn(q, k, v, key_lens=key_lens, key_mask=key_mask, scale=scale)
        ctx.save_for_backward(q, k, v, out, lse, key_lens, key_mask)
        ctx.scale = scale
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse, key_lens, key_mask = ctx.saved_tensors
        dq, dk, dv = cross_attn_bwd(_rows(dout), q, k, v, out, lse, key_lens=key_lens, key_mask=key_mask,
                                    scale=ctx.scale)
        return dq, dk, dv, None, None, None


class _RelBiasAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, table, key_lens, key_mask, kw):
        out, lse = rel_bias_attn(q, k, v, table, key_lens=key_lens, key_mask=key_mask, **kw)
        ctx.save_for_backward(q, k, v, table, out, lse, key_lens, key_mask)
        ctx.kw = kw
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, table, out, lse, key_lens, key_mask = ctx.saved_tensors
        grads = rel_bias_attn_bwd(_rows(dout), q, k, v, table, out, lse, key_lens=key_lens, key_mask=key_mask, **ctx.kw)
        return (*grads, None, None, None)


def cross_attention(q, k, v, *, key_lens=None, key_mask=None, scale: Optional[float] = None):
    """The output of :func:`cross_attn`, differentiable (once) in q, k and v."""
    return _CrossAttention.apply(q, k, v, key_lens, key_mask, scale)


def rel_bias_attention(q, k, v, table, *, max_distance: int = 128, bidirectional: bool = True, causal: bool = False,
                       q_offset: Union[int, str] = 0, key_lens=None, key_mask=None, scale: Optional[float] = None):
    """The output of :func:`rel_bias_attn`, differentiable (once) in q, k, v and the
    table."""
    kw = dict(max_distance=max_distance, bidirectional=bidirectional, causal=causal, q_offset=q_offset, scale=scale)
    return _RelBiasAttention.apply(q, k, v, table, key_lens, key_mask, kw)


def _declare(lib):
    """Argument types of the library's calls."""
    P, R, vp, sz = ctypes.POINTER(_CrossProblem), ctypes.POINTER(_RelBias), ctypes.c_void_p, ctypes.c_size_t
    for name, args in (("cross_attn", [P]), ("rel_bias_attn", [P, R])):
        for b, n in (("", 7 if len(args) == 1 else 8), ("_bwd", 11 if len(args) == 1 else 13)):
            fn = getattr(lib, f"adaspa_{name}{b}_workspace")
            fn.restype, fn.argtypes = sz, args
            fn = getattr(lib, f"adaspa_{name}{b}")
            fn.restype, fn.argtypes = ctypes.c_int, args + [vp] * n + [vp, sz, vp]
