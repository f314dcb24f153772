"""ctypes binding of the key-value cache's operators (see include/tman.h): a cache in pages, the rotation and append of new
tokens, attention of single tokens and of prompts, and eviction by accumulated weight.

Argument marshalling only.  Sizes and strides come from the tensors; a tensor that cannot be what the call takes (type, number of
dimensions, heads that are not contiguous) raises ``TmanError`` before the library is called, everything else is checked there.
"""
from __future__ import annotations

import ctypes as C

from . import api
from .api import TmanError, _check, _ptr, _stream

TMAN_TYPE_F16, TMAN_TYPE_BF16 = 0, 1
_ERR_NULL, _ERR_SHAPE, _ERR_CACHE = -1, -4, -9


class _CCache(C.Structure):
    _fields_ = [("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("page_table", C.c_void_p), ("n_pages", C.c_int32),
                ("n_seqs", C.c_int32), ("max_pages", C.c_int32), ("kv_heads", C.c_int32), ("page", C.c_int32),
                ("dim", C.c_int32), ("type", C.c_int32)]


class _CRope(C.Structure):
    _fields_ = [("cos_sin", C.c_void_p), ("n_pos", C.c_int32), ("rot", C.c_int32), ("axes", C.c_int32),
                ("sections", C.c_int32 * 3), ("interleaved", C.c_int32)]


class _CAttn(C.Structure):
    _fields_ = [("heads", C.c_int32), ("window", C.c_int32), ("scale", C.c_float), ("cap", C.c_float), ("slopes", C.c_void_p)]


# What the checks of every call compare with, looked up once (torch is imported with the first cache, not with this module).
_types, _int32, _float32 = {}, None, None


def _learn_types() -> None:
    global _int32, _float32
    import torch

    _types.update({torch.float16: TMAN_TYPE_F16, torch.bfloat16: TMAN_TYPE_BF16})
    _int32, _float32 = torch.int32, torch.float32


def _wants(ok: bool, where: str, status: int = _ERR_SHAPE) -> None:
    if not ok:
        raise TmanError(status, where)


def _is(t, dtype) -> bool:
    return t.dtype is dtype and t.is_contiguous()


_functions = None


def _load():
    global _functions
    if _functions is None:
        L = api._load()
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        L.tman_rope_append.restype = C.c_int
        L.tman_rope_append.argtypes = [vp, vp, i32, i32, vp, i64, vp, vp, i64, vp, vp, vp, vp, i64, vp, vp]
        L.tman_attn_decode_workspace_bytes.restype = sz
        L.tman_attn_decode_workspace_bytes.argtypes = [vp, vp, i32, i32]
        L.tman_attn_decode.restype = C.c_int
        L.tman_attn_decode.argtypes = [vp, vp, vp, i64, vp, vp, i32, vp, i64, vp, vp, vp, sz, vp]
        L.tman_attn_prefill_workspace_bytes.restype = sz
        L.tman_attn_prefill_workspace_bytes.argtypes = [vp, vp, i32, i32]
        L.tman_attn_prefill.restype = C.c_int
        L.tman_attn_prefill.argtypes = [vp, vp, i32, vp, i64, vp, vp, vp, vp, i32, vp, i64, vp, vp, sz, vp]
        L.tman_kv_evict.restype = C.c_int
        L.tman_kv_evict.argtypes = [vp, vp, vp, i32, i32, i32, vp, i32, vp, vp, vp]
        _functions = L
    return _functions


class KvCache:
    """``tman_kv_cache_t`` over tensors: k_pages, v_pages [n_pages][kv_heads][page][dim] (fp16 or bf16, contiguous), page_table
    int32 [n_seqs][max_pages].  Keeps the tensors alive; holds no state of its own."""

    def __init__(self, k_pages, v_pages, page_table):
        where = "KvCache"
        if not _types:
            _learn_types()
        _wants(k_pages.dim() == 4 and k_pages.shape == v_pages.shape and k_pages.is_contiguous() and v_pages.is_contiguous(), where)
        kind = _types.get(k_pages.dtype, -1)
        _wants(kind >= 0 and v_pages.dtype == k_pages.dtype, where, _ERR_CACHE)
        _wants(page_table.dim() == 2 and _is(page_table, _int32), where)
        self.k_pages, self.v_pages, self.page_table = k_pages, v_pages, page_table
        n_pages, self.kv_heads, self.page, self.dim = k_pages.shape
        self.n_seqs, self.max_pages = page_table.shape
        self.dtype, self.n_pages = k_pages.dtype, n_pages
        self._c = _CCache(_ptr(k_pages), _ptr(v_pages), _ptr(page_table), n_pages, self.n_seqs, self.max_pages, self.kv_heads,
                          self.page, self.dim, kind)
        self._ref = C.byref(self._c)

    def _rows(self, t, where: str, heads: int, tokens: int) -> int:
        """Stride between tokens of t [tokens][heads][dim], whose heads must be contiguous."""
        dim = self.dim
        if t is None or t.shape != (tokens, heads, dim) or t.dtype is not self.dtype:
            raise TmanError(_ERR_NULL if t is None else _ERR_SHAPE if t.shape != (tokens, heads, dim) else _ERR_CACHE, where)
        stride, head, element = t.stride()
        if element != 1 or (head != dim and heads != 1):
            raise TmanError(_ERR_SHAPE, where)
        return heads * dim if tokens == 1 else stride  # (of one token torch may keep any)

    def _weights(self, t, where: str) -> int:
        _wants(t.shape == self.k_pages.shape[:3] and _is(t, _float32), where)
        return t.data_ptr()


class Rope:
    """``tman_rope_t``: cos_sin fp32 [n_pos][rot / 2][2]; sections: pairs per axis of positions (None: one axis)."""

    def __init__(self, cos_sin, sections=None, interleaved: bool = False):
        if not _types:
            _learn_types()
        _wants(cos_sin.dim() == 3 and cos_sin.shape[2] == 2 and _is(cos_sin, _float32), "Rope")
        self.cos_sin = cos_sin
        pairs = cos_sin.shape[1]
        self.sections = tuple(sections) if sections is not None else (pairs,)
        _wants(1 <= len(self.sections) <= 3, "Rope")
        self._c = _CRope(_ptr(cos_sin), cos_sin.shape[0], 2 * pairs, len(self.sections), (C.c_int32 * 3)(*self.sections),
                         1 if interleaved else 0)
        self._ref = C.byref(self._c)


class Attn:
    """``tman_attn_t``: how scores are made and what a window hides; slopes fp32 [heads] on the device or None."""

    def __init__(self, heads: int, scale: float, cap: float = 0.0, window: int = 0, slopes=None):
        if not _types:
            _learn_types()
        _wants(slopes is None or (slopes.dim() == 1 and slopes.shape[0] == heads and _is(slopes, _float32)), "Attn")
        self.heads, self.scale, self.cap, self.window, self.slopes = heads, scale, cap, window, slopes
        self._c = _CAttn(heads, window, scale, cap, _ptr(slopes))
        self._ref = C.byref(self._c)


def _ints(t, n: int, where: str) -> int:
    """Pointer to n int32 numbers."""
    if t is None:
        raise TmanError(_ERR_NULL, where)
    if t.dtype is not _int32 or t.numel() != n or not t.is_contiguous():
        raise TmanError(_ERR_SHAPE, where)
    return t.data_ptr()


def _floats(t, n: int, where: str) -> int:
    if t.dtype is not _float32 or t.numel() != n or not t.is_contiguous():
        raise TmanError(_ERR_SHAPE, where)
    return t.data_ptr()


def _append_args(where, cache, q, k, v, lens, q_out, rope, positions, q_start, weights):
    if k is None:
        raise TmanError(_ERR_NULL, where)
    n, B = k.shape[0], cache.n_seqs
    kv_stride = cache._rows(k, where, cache.kv_heads, n)
    if cache._rows(v, where, cache.kv_heads, n) != kv_stride:
        raise TmanError(_ERR_SHAPE, where)
    heads = q_stride = q_out_stride = 0
    if q is not None:
        heads = q.shape[1]
        q_stride, q_out_stride = cache._rows(q, where, heads, n), cache._rows(q_out, where, heads, n)
    if positions is not None and rope is None:
        raise TmanError(_ERR_SHAPE, where)
    return (cache._ref, None if rope is None else rope._ref, heads, n, None if q is None else q.data_ptr(), q_stride, k.data_ptr(),
            v.data_ptr(), kv_stride, None if positions is None else _ints(positions, len(rope.sections) * n, where),
            None if q_start is None else _ints(q_start, B + 1, where), _ints(lens, B, where),
            None if q_out is None else q_out.data_ptr(), q_out_stride, None if weights is None else cache._weights(weights, where))


def tman_rope_append(cache: KvCache, q, k, v, lens, q_out, rope: Rope = None, positions=None, q_start=None, weights=None,
                     stream=None) -> None:
    """Rotates q and k (q_out may be q; both None: no queries) and writes k and v [n_tokens][kv_heads][dim] into the cache as the
    last positions of their sequences; q_start None: one token a sequence.  k and v have the same distance between tokens."""
    where = "tman_rope_append"
    L = _functions or _load()
    _check(L.tman_rope_append(*_append_args(where, cache, q, k, v, lens, q_out, rope, positions, q_start, weights), _stream(stream)), where)


def bound_rope_append(cache: KvCache, q, k, v, lens, q_out, rope: Rope = None, positions=None, q_start=None, weights=None):
    """The same, checked and marshalled once for calls that run every step with the same tensors: call(stream_handle).  The call keeps
    the tensors and handles alive."""
    where = "tman_rope_append"
    fn, args = _load().tman_rope_append, _append_args(where, cache, q, k, v, lens, q_out, rope, positions, q_start, weights)

    def call(stream_handle):
        _check(fn(*args, stream_handle), where)

    call.holds = (cache, q, k, v, lens, q_out, rope, positions, q_start, weights)  # args are their addresses
    return call


def tman_attn_decode_workspace_bytes(cache: KvCache, attn: Attn, max_len: int, weights: bool = False) -> int:
    return int(_load().tman_attn_decode_workspace_bytes(cache._ref, attn._ref, max_len, 1 if weights else 0))


def _decode_args(where, cache, attn, q, lens, out, max_len, workspace, first, lse, weights):
    B, H = cache.n_seqs, attn.heads
    return (cache._ref, attn._ref, None if q is None else q.data_ptr(), cache._rows(q, where, H, B), _ints(lens, B, where),
            None if first is None else _ints(first, B, where), max_len, None if out is None else out.data_ptr(),
            cache._rows(out, where, H, B), None if lse is None else _floats(lse, B * H, where),
            None if weights is None else cache._weights(weights, where), None if workspace is None else workspace.data_ptr(),
            0 if workspace is None else workspace.nbytes)


def tman_attn_decode(cache: KvCache, attn: Attn, q, lens, out, max_len: int, workspace, first=None, lse=None, weights=None,
                     stream=None) -> None:
    """Attention of one new token of every sequence over its cache; the workspace is zero-filled once by the caller."""
    where = "tman_attn_decode"
    L = _functions or _load()
    _check(L.tman_attn_decode(*_decode_args(where, cache, attn, q, lens, out, max_len, workspace, first, lse, weights), _stream(stream)), where)


def bound_attn_decode(cache: KvCache, attn: Attn, q, lens, out, max_len: int, workspace, first=None, lse=None, weights=None):
    """The same, checked and marshalled once; max_len bounds the lengths of all the steps: call(stream_handle).  The call keeps the
    tensors and handles alive."""
    where = "tman_attn_decode"
    fn, args = _load().tman_attn_decode, _decode_args(where, cache, attn, q, lens, out, max_len, workspace, first, lse, weights)

    def call(stream_handle):
        _check(fn(*args, stream_handle), where)

    call.holds = (cache, attn, q, lens, out, workspace, first, lse, weights)  # args are their addresses
    return call


def tman_attn_prefill_workspace_bytes(cache: KvCache, attn: Attn, n_tokens: int, max_len: int) -> int:
    return int(_load().tman_attn_prefill_workspace_bytes(cache._ref, attn._ref, n_tokens, max_len))


def tman_attn_prefill(cache: KvCache, attn: Attn, q, q_start, lens, out, max_len: int, workspace=None, first=None, end=None, lse=None,
                      stream=None) -> None:
    """Attention of the new tokens of prompts over the cache that holds them; token n sees positions first[n] <= j < end[n].  A tight
    max_len makes the call faster."""
    where = "tman_attn_prefill"
    _wants(q is not None, where, _ERR_NULL)
    n, B, H = q.shape[0], cache.n_seqs, attn.heads
    L = _functions or _load()
    _check(L.tman_attn_prefill(cache._ref, attn._ref, n, q.data_ptr(), cache._rows(q, where, H, n), _ints(q_start, B + 1, where),
                               _ints(lens, B, where), None if first is None else _ints(first, n, where),
                               None if end is None else _ints(end, n, where), max_len, None if out is None else out.data_ptr(),
                               cache._rows(out, where, H, n), None if lse is None else _floats(lse, n * H, where),
                               None if workspace is None else workspace.data_ptr(), 0 if workspace is None else workspace.nbytes,
                               _stream(stream)), where)


def tman_kv_evict(cache: KvCache, weights, lens, keep: int, recent: int, new_table, new_lens, kept, max_len: int, stream=None) -> None:
    """Keeps `keep` positions of every sequence and key-value head (the `recent` last and the largest weights) in the pages of
    new_table; new_lens [n_seqs] (lens itself will do) and kept [n_seqs][kv_heads][keep] receive the lengths and the positions that stayed."""
    where = "tman_kv_evict"
    _wants(weights is not None and new_table is not None, where, _ERR_NULL)
    B = cache.n_seqs
    _wants(new_table.dim() == 2 and new_table.shape[0] == B, where)
    pages = new_table.shape[1]
    L = _functions or _load()
    _check(L.tman_kv_evict(cache._ref, cache._weights(weights, where), _ints(lens, B, where), keep, recent, max_len,
                           _ints(new_table, B * pages, where), pages, _ints(new_lens, B, where),
                           _ints(kept, B * cache.kv_heads * keep, where), _stream(stream)), where)
