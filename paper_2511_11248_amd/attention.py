"""ctypes binding of the key-value cache's operators (see include/tman.h): a cache in pages, of 16 bits or 8, the pages of a step, the
norm, rotation and append of new tokens, attention of single tokens and of prompts, and eviction by accumulated weight.

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


class _CNorm(C.Structure):
    _fields_ = [("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("eps", C.c_float), ("per_head", C.c_int32)]


class _CCache8(C.Structure):
    _fields_ = [("pages", _CCache), ("k_exps", C.c_void_p), ("v_exps", C.c_void_p)]


class _CAttn(C.Structure):
    _fields_ = [("heads", C.c_int32), ("window", C.c_int32), ("scale", C.c_float), ("cap", C.c_float), ("slopes", C.c_void_p)]


# What the checks of every call compare with, looked up once (torch is imported with the first cache, not with this module).
_types, _int32, _int64, _float32, _uint8, _code = {}, None, None, None, None, None


def _learn_types() -> None:
    global _int32, _int64, _float32, _uint8, _code
    import torch

    _int64, _uint8, _code = torch.int64, torch.uint8, torch.float8_e4m3fn

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
        L.tman_norm_rope_append.restype = C.c_int
        L.tman_norm_rope_append.argtypes = [vp, vp, vp, i32, i32, vp, i64, vp, vp, i64, vp, vp, vp, vp, i64, vp, vp]
        L.tman_kv8_append.restype = C.c_int
        L.tman_kv8_append.argtypes = [vp, vp, vp, i32, i32, vp, i64, vp, vp, i64, vp, vp, vp, vp, i64, vp]
        L.tman_attn_decode_kv8_workspace_bytes.restype = sz
        L.tman_attn_decode_kv8_workspace_bytes.argtypes = [vp, vp, i32]
        L.tman_attn_decode_kv8.restype = C.c_int
        L.tman_attn_decode_kv8.argtypes = [vp, vp, vp, i64, vp, vp, i32, vp, i64, vp, vp, sz, vp]
        L.tman_attn_prefill_kv8_workspace_bytes.restype = sz
        L.tman_attn_prefill_kv8_workspace_bytes.argtypes = [vp, vp, i32, i32]
        L.tman_attn_prefill_kv8.restype = C.c_int
        L.tman_attn_prefill_kv8.argtypes = [vp, vp, i32, vp, i64, vp, vp, vp, vp, i32, vp, i64, vp, vp, sz, vp]
        L.tman_kv_plan_workspace_bytes.restype = sz
        L.tman_kv_plan_workspace_bytes.argtypes = [i32, i32]
        L.tman_kv_plan.restype = C.c_int
        L.tman_kv_plan.argtypes = [vp, i32, i32, i32, vp, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        _functions = L
    return _functions


class KvCache:
    """``tman_kv_cache_t`` over tensors: k_pages, v_pages [n_pages][kv_heads][page][dim] (fp16 or bf16, contiguous), page_table
    int32 [n_seqs][max_pages].  Keeps the tensors alive; holds no state of its own."""

    _codes = False  # (looked at in every call: 0.1 us less than isinstance in a call of its own)

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


class KvCache8(KvCache):
    """``tman_kv8_cache_t`` over tensors: k_pages, v_pages [n_pages][kv_heads][page][dim] of e4m3 codes (float8_e4m3fn or uint8),
    k_exps, v_exps uint8 [n_pages][kv_heads][page / 16], page_table int32 [n_seqs][max_pages]; dtype (fp16 or bf16) of queries, new
    keys and values, and outputs.  Keeps the tensors alive; holds no state of its own."""

    _codes = True

    def __init__(self, k_pages, v_pages, k_exps, v_exps, page_table, dtype):
        where = "KvCache8"
        if not _types:
            _learn_types()
        _wants(k_pages.dim() == 4 and k_pages.shape == v_pages.shape and k_pages.is_contiguous() and v_pages.is_contiguous(), where)
        kind = _types.get(dtype, -1)
        _wants(kind >= 0 and k_pages.dtype in (_code, _uint8) and v_pages.dtype in (_code, _uint8), where, _ERR_CACHE)
        _wants(page_table.dim() == 2 and _is(page_table, _int32), where)
        n_pages, self.kv_heads, self.page, self.dim = k_pages.shape
        blocks = (n_pages, self.kv_heads, self.page // 16)
        _wants(k_exps.shape == blocks and v_exps.shape == blocks and _is(k_exps, _uint8) and _is(v_exps, _uint8), where)
        self.k_pages, self.v_pages, self.k_exps, self.v_exps, self.page_table = k_pages, v_pages, k_exps, v_exps, page_table
        self.n_seqs, self.max_pages = page_table.shape
        self.dtype, self.n_pages = dtype, n_pages
        self._c = _CCache8(_CCache(_ptr(k_pages), _ptr(v_pages), _ptr(page_table), n_pages, self.n_seqs, self.max_pages, self.kv_heads,
                                   self.page, self.dim, kind), _ptr(k_exps), _ptr(v_exps))
        self._ref = C.byref(self._c)


def _of_8_bits(cache, where: str) -> None:
    _wants(isinstance(cache, KvCache8), where, _ERR_CACHE)


class HeadNorm:
    """``tman_head_norm_t``: weights fp32 [dim], or [heads][dim] of queries and [kv_heads][dim] of keys, or None for ones."""

    def __init__(self, q_weight, k_weight, eps: float):
        if not _types:
            _learn_types()
        given = [w for w in (q_weight, k_weight) if w is not None]
        _wants(all(w.dim() == given[0].dim() and w.dim() in (1, 2) and _is(w, _float32) for w in given), "HeadNorm")
        self.q_weight, self.k_weight, self.eps = q_weight, k_weight, eps
        per_head = bool(given) and given[0].dim() == 2
        # what they are for, looked at once: (heads of queries or None, of keys or None, dims)
        self._heads = tuple(w.shape[0] if per_head and w is not None else None for w in (q_weight, k_weight))
        self._dims = {w.shape[-1] for w in given}
        _wants(len(self._dims) <= 1, "HeadNorm")
        self._c = _CNorm(_ptr(q_weight), _ptr(k_weight), eps, 1 if per_head else 0)
        self._ref = C.byref(self._c)

    def _fits(self, heads: int, cache, where: str) -> None:
        q, k = self._heads
        if (q is not None and q != heads and heads) or (k is not None and k != cache.kv_heads) or (self._dims and cache.dim not in self._dims):
            raise TmanError(_ERR_SHAPE, where)


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
    if cache._codes:
        raise TmanError(_ERR_CACHE, where)
    L = _functions or _load()
    _check(L.tman_rope_append(*_append_args(where, cache, q, k, v, lens, q_out, rope, positions, q_start, weights), _stream(stream)), where)


def bound_rope_append(cache: KvCache, q, k, v, lens, q_out, rope: Rope = None, positions=None, q_start=None, weights=None):
    """The same, checked and marshalled once for calls that run every step with the same tensors: call(stream_handle).  The call keeps
    the tensors and handles alive."""
    where = "tman_rope_append"
    if cache._codes:
        raise TmanError(_ERR_CACHE, where)
    fn, args = _load().tman_rope_append, _append_args(where, cache, q, k, v, lens, q_out, rope, positions, q_start, weights)

    def call(stream_handle):
        _check(fn(*args, stream_handle), where)

    call.holds = (cache, q, k, v, lens, q_out, rope, positions, q_start, weights)  # args are their addresses
    return call


def _normed(args, norm, heads, cache, where):
    """The arguments of an append with a norm ahead of the rotation."""
    if norm is not None:
        norm._fits(heads, cache, where)
    return (args[0], None if norm is None else norm._ref, *args[1:])


def tman_norm_rope_append(cache: KvCache, norm: HeadNorm, q, k, v, lens, q_out, rope: Rope = None, positions=None, q_start=None,
                          weights=None, stream=None) -> None:
    """tman_rope_append with the norm of query and key heads in the same pass."""
    where = "tman_norm_rope_append"
    if cache._codes:
        raise TmanError(_ERR_CACHE, where)
    _wants(norm is not None, where, _ERR_NULL)
    L = _functions or _load()
    args = _append_args(where, cache, q, k, v, lens, q_out, rope, positions, q_start, weights)
    _check(L.tman_norm_rope_append(*_normed(args, norm, args[2], cache, where), _stream(stream)), where)


def tman_kv8_append(cache: KvCache8, q, k, v, lens, q_out, norm: HeadNorm = None, rope: Rope = None, positions=None, q_start=None,
                    stream=None) -> None:
    """The same (norm None: without one) into a cache held in 8 bits."""
    where = "tman_kv8_append"
    _of_8_bits(cache, where)
    L = _functions or _load()
    args = _append_args(where, cache, q, k, v, lens, q_out, rope, positions, q_start, None)
    _check(L.tman_kv8_append(*_normed(args[:-1], norm, args[2], cache, where), _stream(stream)), where)


def bound_kv8_append(cache: KvCache8, q, k, v, lens, q_out, norm: HeadNorm = None, rope: Rope = None, positions=None, q_start=None):
    """The same, checked and marshalled once: call(stream_handle).  The call keeps the tensors and handles alive."""
    where = "tman_kv8_append"
    _of_8_bits(cache, where)
    args = _append_args(where, cache, q, k, v, lens, q_out, rope, positions, q_start, None)
    fn, args = _load().tman_kv8_append, _normed(args[:-1], norm, args[2], cache, where)

    def call(stream_handle):
        _check(fn(*args, stream_handle), where)

    call.holds = (cache, q, k, v, lens, q_out, norm, rope, positions, q_start)  # args are their addresses
    return call


def tman_attn_decode_workspace_bytes(cache: KvCache, attn: Attn, max_len: int, weights: bool = False) -> int:
    if cache._codes:
        raise TmanError(_ERR_CACHE, "tman_attn_decode_workspace_bytes")
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
    if cache._codes:
        raise TmanError(_ERR_CACHE, where)
    L = _functions or _load()
    _check(L.tman_attn_decode(*_decode_args(where, cache, attn, q, lens, out, max_len, workspace, first, lse, weights), _stream(stream)), where)


def bound_attn_decode(cache: KvCache, attn: Attn, q, lens, out, max_len: int, workspace, first=None, lse=None, weights=None):
    """The same, checked and marshalled once; max_len bounds the lengths of all the steps: call(stream_handle).  The call keeps the
    tensors and handles alive."""
    where = "tman_attn_decode"
    if cache._codes:
        raise TmanError(_ERR_CACHE, where)
    fn, args = _load().tman_attn_decode, _decode_args(where, cache, attn, q, lens, out, max_len, workspace, first, lse, weights)

    def call(stream_handle):
        _check(fn(*args, stream_handle), where)

    call.holds = (cache, attn, q, lens, out, workspace, first, lse, weights)  # args are their addresses
    return call


def tman_attn_decode_kv8_workspace_bytes(cache: KvCache8, attn: Attn, max_len: int) -> int:
    _of_8_bits(cache, "tman_attn_decode_kv8_workspace_bytes")
    return int(_load().tman_attn_decode_kv8_workspace_bytes(cache._ref, attn._ref, max_len))


def _decode8_args(*args):
    a = _decode_args(*args, None)
    return a[:10] + a[11:]  # no weights


def tman_attn_decode_kv8(cache: KvCache8, attn: Attn, q, lens, out, max_len: int, workspace, first=None, lse=None, stream=None) -> None:
    """tman_attn_decode over a cache held in 8 bits."""
    where = "tman_attn_decode_kv8"
    _of_8_bits(cache, where)
    L = _functions or _load()
    _check(L.tman_attn_decode_kv8(*_decode8_args(where, cache, attn, q, lens, out, max_len, workspace, first, lse), _stream(stream)), where)


def bound_attn_decode_kv8(cache: KvCache8, attn: Attn, q, lens, out, max_len: int, workspace, first=None, lse=None):
    """The same, checked and marshalled once; max_len bounds the lengths of all the steps: call(stream_handle).  The call keeps the
    tensors and handles alive."""
    where = "tman_attn_decode_kv8"
    _of_8_bits(cache, where)
    fn, args = _load().tman_attn_decode_kv8, _decode8_args(where, cache, attn, q, lens, out, max_len, workspace, first, lse)

    def call(stream_handle):
        _check(fn(*args, stream_handle), where)

    call.holds = (cache, attn, q, lens, out, workspace, first, lse)  # args are their addresses
    return call


def tman_attn_prefill_workspace_bytes(cache: KvCache, attn: Attn, n_tokens: int, max_len: int) -> int:
    if cache._codes:
        raise TmanError(_ERR_CACHE, "tman_attn_prefill_workspace_bytes")
    return int(_load().tman_attn_prefill_workspace_bytes(cache._ref, attn._ref, n_tokens, max_len))


def _prefill(fn, where, cache, attn, q, q_start, lens, out, max_len, workspace, first, end, lse, stream):
    _wants(q is not None, where, _ERR_NULL)
    n, B, H = q.shape[0], cache.n_seqs, attn.heads
    _check(fn(cache._ref, attn._ref, n, q.data_ptr(), cache._rows(q, where, H, n), _ints(q_start, B + 1, where), _ints(lens, B, where),
              None if first is None else _ints(first, n, where), None if end is None else _ints(end, n, where), max_len,
              None if out is None else out.data_ptr(), cache._rows(out, where, H, n), None if lse is None else _floats(lse, n * H, where),
              None if workspace is None else workspace.data_ptr(), 0 if workspace is None else workspace.nbytes, _stream(stream)), where)


def tman_attn_prefill(cache: KvCache, attn: Attn, q, q_start, lens, out, max_len: int, workspace=None, first=None, end=None, lse=None,
                      stream=None) -> None:
    """Attention of the new tokens of prompts over the cache that holds them; token n sees positions first[n] <= j < end[n].  A tight
    max_len makes the call faster."""
    where = "tman_attn_prefill"
    if cache._codes:
        raise TmanError(_ERR_CACHE, where)
    L = _functions or _load()
    _prefill(L.tman_attn_prefill, where, cache, attn, q, q_start, lens, out, max_len, workspace, first, end, lse, stream)


def tman_attn_prefill_kv8_workspace_bytes(cache: KvCache8, attn: Attn, n_tokens: int, max_len: int) -> int:
    _of_8_bits(cache, "tman_attn_prefill_kv8_workspace_bytes")
    return int(_load().tman_attn_prefill_kv8_workspace_bytes(cache._ref, attn._ref, n_tokens, max_len))


def tman_attn_prefill_kv8(cache: KvCache8, attn: Attn, q, q_start, lens, out, max_len: int, workspace=None, first=None, end=None,
                          lse=None, stream=None) -> None:
    """tman_attn_prefill over a cache held in 8 bits.  A tight max_len makes the call faster, and the workspace smaller."""
    where = "tman_attn_prefill_kv8"
    _of_8_bits(cache, where)
    L = _functions or _load()
    _prefill(L.tman_attn_prefill_kv8, where, cache, attn, q, q_start, lens, out, max_len, workspace, first, end, lse, stream)


def tman_kv_evict(cache: KvCache, weights, lens, keep: int, recent: int, new_table, new_lens, kept, max_len: int, stream=None) -> None:
    """Keeps `keep` positions of every sequence and key-value head (the `recent` last and the largest weights) in the pages of
    new_table; new_lens [n_seqs] (lens itself will do) and kept [n_seqs][kv_heads][keep] receive the lengths and the positions that stayed."""
    where = "tman_kv_evict"
    if cache._codes:
        raise TmanError(_ERR_CACHE, where)
    _wants(weights is not None and new_table is not None, where, _ERR_NULL)
    B = cache.n_seqs
    _wants(new_table.dim() == 2 and new_table.shape[0] == B, where)
    pages = new_table.shape[1]
    L = _functions or _load()
    _check(L.tman_kv_evict(cache._ref, cache._weights(weights, where), _ints(lens, B, where), keep, recent, max_len,
                           _ints(new_table, B * pages, where), pages, _ints(new_lens, B, where),
                           _ints(kept, B * cache.kv_heads * keep, where), _stream(stream)), where)


def tman_kv_plan_workspace_bytes(n_seqs: int, n_tokens: int) -> int:
    return int(_load().tman_kv_plan_workspace_bytes(n_seqs, n_tokens))


def _plan_args(where, page_table, page, lens, more, free_pages, free_left, new_lens, new_left, q_start, slots, positions, owners, workspace,
               n_tokens):
    if not _types:
        _learn_types()
    if page_table is None or free_pages is None:
        raise TmanError(_ERR_NULL, where)
    table, stack = page_table.shape, free_pages.shape
    if len(table) != 2 or len(stack) != 1 or not _is(page_table, _int32) or not _is(free_pages, _int32):
        raise TmanError(_ERR_SHAPE, where)
    B, wide = table
    if n_tokens is None:
        given = slots if slots is not None else positions if positions is not None else owners
        if given is None:
            raise TmanError(_ERR_SHAPE, where)
        n_tokens = given.numel()
    if slots is not None and (slots.dtype is not _int64 or slots.numel() != n_tokens or not slots.is_contiguous()):
        raise TmanError(_ERR_SHAPE, where)
    i32 = _int32
    # what _ints would check of each, in one expression (a call of a few microseconds)
    if lens is None or more is None or free_left is None or new_lens is None or new_left is None or q_start is None or not (
            lens.dtype is more.dtype is free_left.dtype is new_lens.dtype is new_left.dtype is q_start.dtype is i32
            and lens.numel() == more.numel() == new_lens.numel() == B and free_left.numel() == new_left.numel() == 1
            and q_start.numel() == B + 1 and lens.is_contiguous() and more.is_contiguous() and new_lens.is_contiguous()
            and q_start.is_contiguous()):
        raise TmanError(_ERR_NULL if any(t is None for t in (lens, more, free_left, new_lens, new_left, q_start)) else _ERR_SHAPE, where)
    return (page_table.data_ptr(), B, wide, page, lens.data_ptr(), more.data_ptr(), free_pages.data_ptr(), stack[0], free_left.data_ptr(),
            n_tokens, new_lens.data_ptr(), new_left.data_ptr(), q_start.data_ptr(), None if slots is None else slots.data_ptr(),
            None if positions is None else _ints(positions, n_tokens, where), None if owners is None else _ints(owners, n_tokens, where),
            None if workspace is None else workspace.data_ptr(), 0 if workspace is None else workspace.nbytes)


def tman_kv_plan(page_table, page: int, lens, more, free_pages, free_left, new_lens, new_left, q_start, slots=None, positions=None,
                 owners=None, workspace=None, n_tokens: int = None, stream=None) -> None:
    """Gives pages of `page` positions to the sequences that grow, takes back those of the ones that shrink, and writes the places of the
    new tokens; n_tokens, the most that are granted, is what slots, positions and owners hold."""
    where = "tman_kv_plan"
    L = _functions or _load()
    _check(L.tman_kv_plan(*_plan_args(where, page_table, page, lens, more, free_pages, free_left, new_lens, new_left, q_start, slots,
                                      positions, owners, workspace, n_tokens), _stream(stream)), where)


def bound_kv_plan(page_table, page: int, lens, more, free_pages, free_left, new_lens, new_left, q_start, slots=None, positions=None,
                  owners=None, workspace=None, n_tokens: int = None):
    """The same, checked and marshalled once: call(stream_handle).  The call keeps the tensors alive."""
    where = "tman_kv_plan"
    fn, args = _load().tman_kv_plan, _plan_args(where, page_table, page, lens, more, free_pages, free_left, new_lens, new_left, q_start, slots,
                                                positions, owners, workspace, n_tokens)

    def call(stream_handle):
        _check(fn(*args, stream_handle), where)

    call.holds = (page_table, lens, more, free_pages, free_left, new_lens, new_left, q_start, slots, positions, owners, workspace)
    return call
