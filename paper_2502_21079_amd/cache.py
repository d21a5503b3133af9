"""A key/value cache held in 8 bits: quantising tokens as they are written,
reading them back, and attention over the cache as it lies.

Argument marshalling only, as in the package's other calls: every step runs in
the HIP kernels of ``libadaspa.so`` (the C ABI is in ``include/adaspa.h``).

* :class:`KVCache`, :func:`kv_cache`    a pool of pages
* :func:`cache_write`                   new keys and values into their pages
* :func:`cache_read`                    whole sequences, or parts, in 16 bits again
* :func:`cache_attn`                    attention of new queries (single tokens or
      whole prompts) over a sequence's pages

A page holds ``page`` tokens of one sequence for every key head, with a scale for
each head's keys and one for its values.  ``page_table`` (int32 [B, max_pages])
names the pages of each sequence in order; ``lens`` (int32 [B]) counts its tokens.
Sequences may share pages that are only read.  Table and lengths stay on the GPU, so
a captured graph follows them as they change.
"""
from __future__ import annotations

import ctypes
import functools
from dataclasses import dataclass
from operator import index
from typing import Optional

import torch

from . import AdaspaError, _check, _on, _ptr, _stream, load_library
from .prompt import _DTYPES, _I64x3, _check_like, _check_lse, _contiguous, _new, _new_strides, _scratch, _steps

__all__ = ["KVCache", "kv_cache", "cache_write", "cache_read", "cache_attn", "cache_attn_workspace"]

_E4M3 = torch.float8_e4m3fn
_PAGES = (16, 32, 64, 128)


class _CacheProblem(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("batch", "heads", "kv_heads", "len", "head_dim", "dtype", "pages", "page",
                                               "max_pages", "causal")]
                + [("softmax_scale", ctypes.c_float), ("table_stride", ctypes.c_int64)]
                + [(n + "_stride", _I64x3) for n in ("q", "out", "k", "v")])


class _Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "page_table")]


@dataclass
class KVCache:
    """A pool of pages.  A value is its code times its page's and head's scale, a
    power of two.  (Magnitudes from 248 * 2^120 on, among bf16's last, are rounded to 2^128,
    which is infinite where it is read.)"""
    k: torch.Tensor               # e4m3 [pages, Hk, page, D]
    v: torch.Tensor               # e4m3 [pages, Hk, page / 16, D, 16]: sixteen tokens of a channel side by side
    k_scale: torch.Tensor         # fp32 [pages, Hk]
    v_scale: torch.Tensor         # fp32 [pages, Hk]


def kv_cache(pages: int, kv_heads: int, page: int, head_dim: int, device="cuda") -> KVCache:
    """A new pool.  Its contents need not be set: only tokens that were written are
    ever read."""
    pages, kv_heads, page, head_dim = map(index, (pages, kv_heads, page, head_dim))
    if page not in _PAGES or head_dim not in (64, 128) or pages < 0 or kv_heads < 1:
        raise AdaspaError(f"a page holds {_PAGES} tokens and a head 64 or 128 channels, got {page} and {head_dim}")

    def new(*shape, dtype):
        return torch.empty(shape, dtype=dtype, device=device)
    return KVCache(new(pages, kv_heads, page, head_dim, dtype=_E4M3),
                   new(pages, kv_heads, page // 16, head_dim, 16, dtype=_E4M3),
                   new(pages, kv_heads, dtype=torch.float32), new(pages, kv_heads, dtype=torch.float32))


# --- plans: argument structures and sizes, once per set of values -----------------

class _Plan:
    __slots__ = ("struct", "prob", "need", "rows")


@functools.lru_cache(maxsize=512)
def _pool(k, v, ks, vs):
    """(pages, Hk, page, D) of a pool with these shapes."""
    if len(k) != 4 or k[2] not in _PAGES or v != (k[0], k[1], k[2] // 16, k[3], 16) or ks != k[:2] or vs != k[:2]:
        raise AdaspaError("a cache has k [pages, Hk, page, D], v [pages, Hk, page / 16, D, 16] and scales [pages, Hk], got "
                          f"{tuple(k)}, {tuple(v)}, {tuple(ks)} and {tuple(vs)}")
    return tuple(k)


@functools.lru_cache(maxsize=512)
def _plan(pool, dtype, table, table_step, shape, strides, outs, causal, scale) -> _Plan:
    """Sets up the structure of a call: attention where causal is given (shape and
    strides of q, of out), else reading or writing (strides of k, of v)."""
    pages, Hk, page, D = pool
    B, H, L, d = shape
    if d != D or len(table) != 2 or table[0] != B or (H % Hk if causal is not None else H != Hk):
        raise AdaspaError(f"shapes do not fit: {tuple(shape)} for a cache of {Hk} heads of {D}, page table {tuple(table)}")
    if max(*shape, pages, table[1]) >= 1 << 31:                # the structure's numbers would wrap
        raise AdaspaError("sizes must be below 2^31")
    if table_step[1] != 1 and table[1] > 1:
        raise AdaspaError("the page table's rows must be contiguous")
    p = _CacheProblem(B, H, Hk, L, D, dtype, pages, page, table[1], int(bool(causal)), scale,
                      table_step[0] if B > 1 else 0)
    if causal is None:
        names = ("k", "v")
    else:
        names, strides = ("q", "out"), (strides[0], _new_strides(shape, strides[0]) if outs is None else outs)
    for n, s in zip(names, strides):
        setattr(p, n + "_stride", _I64x3(*_steps(shape, s)))
    plan = _Plan()
    plan.struct, plan.prob, plan.rows = p, ctypes.byref(p), (B, H, L)
    plan.need = 0 if causal is None else int(load_library().adaspa_cache_attn_workspace(plan.prob))
    return plan


# --- argument checks ----------------------------------------------------------------

def _check_cache(cache, table, dev):
    """The pool's sizes and its pointers, after checks of type and device."""
    k, v, ks, vs = cache.k, cache.v, cache.k_scale, cache.v_scale
    if k.dtype is not _E4M3 or v.dtype is not _E4M3 or ks.dtype is not torch.float32 or vs.dtype is not torch.float32:
        raise AdaspaError("a cache has e4m3 codes and fp32 scales")
    for t in (k, v, ks, vs):
        if t.get_device() != dev or not t.is_contiguous():
            raise AdaspaError("a cache's tensors must be contiguous and on the inputs' device")
    if table.dtype is not torch.int32 or table.get_device() != dev:
        raise AdaspaError("page_table must be an int32 [B, max_pages] tensor on the inputs' device")
    return _pool(k.shape, v.shape, ks.shape, vs.shape), \
        ctypes.byref(_Cache(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), table.data_ptr()))


def _check_count(t, name, B, dev):
    if t is not None and (t.dtype is not torch.int32 or t.shape != (B,) or not t.is_contiguous()
                          or t.get_device() != dev):
        raise AdaspaError(f"{name} must be a contiguous int32 [B] = [{B}] tensor on the inputs' device")


def _device_of(t, what):
    dev = t.get_device()
    if dev < 0 or t.dtype not in _DTYPES or t.dim() != 4:
        raise AdaspaError(f"{what} must be bf16 or fp16 CUDA tensors [B, heads, tokens, D]")
    return dev


# --- calls --------------------------------------------------------------------------

def cache_write(k, v, cache: KVCache, page_table, lens, *, new_lens=None) -> None:
    """Writes k, v [B, Hk, T, D] behind the ``lens[b]`` tokens that each sequence
    has in the cache already (``lens`` itself is not changed); ``new_lens`` (int32 [B])
    leaves sample b its first new_lens[b] tokens.

    Each page and head gets the least scale (a power of two, at least 2^-126) that
    takes its largest finite magnitude to at most 448, the largest code; values are
    rounded to the nearest code, ties to even.  A page that holds tokens already keeps
    the larger of its scale and the new tokens'; where it grows, their codes are brought
    to it.  Infinities and NaN are kept as NaN.  Tokens behind the last one stay as they
    were; tokens for pages that the table does not name, or that are not in the pool, are
    dropped, and so are all of a sample with lens[b] < 0.  Pages that are written belong to
    one sequence; the same page twice is an error of the caller's.  A sample without new
    tokens writes nothing, so the table may name another's pages for it."""
    dev = _device_of(k, "k, v")
    if v.dtype is not k.dtype or v.get_device() != dev or v.shape != k.shape:
        raise AdaspaError("k, v must share one type, shape and device")
    pool, ref = _check_cache(cache, page_table, dev)
    _check_count(lens, "lens", k.shape[0], dev)
    _check_count(new_lens, "new_lens", k.shape[0], dev)
    plan = _plan(pool, _DTYPES[k.dtype], page_table.shape, page_table.stride(), k.shape, (k.stride(), v.stride()), None,
                 None, 0.0)
    with _on(dev):
        _check(load_library().adaspa_cache_write(plan.prob, ref, k.data_ptr(), v.data_ptr(), lens.data_ptr(),
                                                 _ptr(new_lens), _stream(k.device)))


def cache_read(cache: KVCache, page_table, lens, tokens: int, *, starts=None, dtype=torch.bfloat16, k=None, v=None):
    """(k, v) [B, Hk, tokens, D] in ``dtype`` (bf16 or fp16): row t of sample b is the
    token at position t, or ``starts[b]`` + t (int32 [B]).  Rows that are not among the
    sequence's ``lens[b]`` tokens, or on a page that is not in the pool, are zeros.  Values are
    exact within the type's range (in fp16 those that were rounded to 2^16 are infinite).  ``k`` and ``v`` are filled where they
    are given; they must not overlap."""
    dev = cache.k.get_device()
    if dtype not in _DTYPES:
        raise AdaspaError(f"dtype must be bf16 or fp16, got {dtype}")
    if dev < 0:
        raise AdaspaError("a cache's tensors must be on a GPU")
    pool, ref = _check_cache(cache, page_table, dev)
    B = page_table.shape[0] if page_table.dim() else 0
    _check_count(lens, "lens", B, dev)
    _check_count(starts, "starts", B, dev)
    shape = (B, pool[1], index(tokens), pool[3])
    if shape[2] < 0:
        raise AdaspaError(f"tokens must not be negative, got {tokens}")
    for t, name in ((k, "k"), (v, "v")):
        if t is not None and (t.dtype is not dtype or t.shape != shape or t.get_device() != dev):
            raise AdaspaError(f"{name} must be a {dtype} tensor of shape {shape} on the cache's device")
    k = torch.empty(shape, dtype=dtype, device=cache.k.device) if k is None else k
    v = torch.empty(shape, dtype=dtype, device=cache.k.device) if v is None else v
    plan = _plan(pool, _DTYPES[dtype], page_table.shape, page_table.stride(), shape, (k.stride(), v.stride()), None, None,
                 0.0)
    with _on(dev):
        _check(load_library().adaspa_cache_read(plan.prob, ref, lens.data_ptr(), _ptr(starts), k.data_ptr(), v.data_ptr(),
                                                _stream(cache.k.device)))
    return k, v


def cache_attn(q, cache: KVCache, page_table, lens, *, q_lens=None, causal: bool = True, scale: Optional[float] = None,
               out=None, lse=None, want_lse: bool = True, workspace=None):
    """Attention of q [B, H, Lq, D] over the ``lens[b]`` tokens of each sequence
    (H % Hk == 0, runs of H / Hk query heads share a key head).  Returns (out, lse).

    The queries are their sequence's last tokens, whose keys and values are in the
    cache already; ``q_lens`` (int32 [B]) leaves sample b its first q_lens[b], the rows behind
    give 0 and an lse of -inf.  With ``causal`` query i sees the tokens up to its own place,
    without it all of the sequence's.  A row that sees no token gives 0 and -inf; tokens behind
    lens[b], or on pages that are not in the pool, take no part, whatever is there; those that
    only the order hides from a row must be finite, as those that it sees.  ``scale``
    defaults to 1 / sqrt(D), which values up to 0 stand for too.  ``workspace`` (at least
    :func:`cache_attn_workspace` bytes, any type) is allocated here when not given and
    needed.  The same arguments give the same bits.  How the tokens are divided over the GPU
    follows the shapes (the page table's width among them) and, up to 48 rows a key head, all
    of ``lens``: in another batch a sequence's results may differ in their last bits."""
    dev = _device_of(q, "q")
    pool, ref = _check_cache(cache, page_table, dev)
    _check_count(lens, "lens", q.shape[0], dev)
    _check_count(q_lens, "q_lens", q.shape[0], dev)
    plan = _plan(pool, _DTYPES[q.dtype], page_table.shape, page_table.stride(), q.shape, (q.stride(),),
                 None if out is None else _check_like(out, q, "out"), bool(causal), 0.0 if scale is None else float(scale))
    if out is None:
        out = _new(q)
    if lse is not None:
        _check_lse(lse, q)
    elif want_lse:
        lse = q.new_empty(plan.rows, dtype=torch.float32)
    workspace, ws_bytes = _scratch(workspace, plan.need, q)
    with _on(dev):
        _check(load_library().adaspa_cache_attn(plan.prob, ref, q.data_ptr(), lens.data_ptr(), _ptr(q_lens),
                                                out.data_ptr(), _ptr(lse), _ptr(workspace), ws_bytes, _stream(q.device)))
    return out, lse


def cache_attn_workspace(q_shape, cache: KVCache, max_pages: int, dtype=torch.bfloat16, *,
                         causal: Optional[bool] = None) -> int:
    """Bytes of the workspace of :func:`cache_attn` for q of this shape and type, a page
    table of this width and this ``causal``; None: as many as serve either."""
    if dtype not in _DTYPES:
        raise AdaspaError(f"dtype must be bf16 or fp16, got {dtype}")
    shape = tuple(map(index, q_shape))
    pool = _pool(cache.k.shape, cache.v.shape, cache.k_scale.shape, cache.v_scale.shape)
    return max(_plan(pool, _DTYPES[dtype], (shape[0], index(max_pages)), (index(max_pages), 1), shape, (_contiguous(shape),),
                     None, order, 0.0).need for order in ((True, False) if causal is None else (bool(causal),)))


def _declare(lib):
    """Argument types of the library's calls."""
    P, C, vp, sz = ctypes.POINTER(_CacheProblem), ctypes.POINTER(_Cache), ctypes.c_void_p, ctypes.c_size_t
    for name, n in (("adaspa_cache_write", 5), ("adaspa_cache_read", 5)):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = ctypes.c_int, [P, C] + [vp] * n
    lib.adaspa_cache_attn_workspace.restype, lib.adaspa_cache_attn_workspace.argtypes = sz, [P]
    lib.adaspa_cache_attn.restype = ctypes.c_int
    lib.adaspa_cache_attn.argtypes = [P, C] + [vp] * 6 + [sz, vp]
