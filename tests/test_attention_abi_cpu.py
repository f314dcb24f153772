"""Host-side checks of the key-value cache's operators: size queries, and refusals before anything is launched."""
import ctypes as C

import pytest
import torch

import paper_2511_11248_amd as tman
from paper_2511_11248_amd import attention as at

FAKE = 0x1000  # non-NULL, 16-byte aligned, never dereferenced: validation fails first
NULL, SHAPE, WORKSPACE, ALIGN, CACHE = -1, -4, -5, -6, -9


def _cache(**over):
    f = dict(k_pages=FAKE, v_pages=FAKE, page_table=FAKE, n_pages=8, n_seqs=2, max_pages=4, kv_heads=2, page=16, dim=64, type=0)
    f.update(over)
    return C.byref(at._CCache(*[f[n] for n, _ in at._CCache._fields_]))


def _attn(heads=4, window=0, scale=1.0, cap=0.0, slopes=None):
    return C.byref(at._CAttn(heads, window, scale, cap, slopes))


def _rope(cos_sin=FAKE, n_pos=8, rot=64, axes=1, sections=(32, 0, 0), interleaved=0):
    return C.byref(at._CRope(cos_sin, n_pos, rot, axes, (C.c_int32 * 3)(*sections), interleaved))


def _append(L, cache, rope=None, heads=4, n=2, q=FAKE, qs=256, k=FAKE, v=FAKE, kvs=128, pos=None, start=None, lens=FAKE, qo=FAKE,
            qos=256, w=None):
    return L.tman_rope_append(cache, rope, heads, n, q, qs, k, v, kvs, pos, start, lens, qo, qos, w, None)


def _decode(L, cache, attn, q=FAKE, qs=256, lens=FAKE, first=None, max_len=64, out=FAKE, os=256, lse=None, w=None, ws=FAKE, wb=1 << 30):
    return L.tman_attn_decode(cache, attn, q, qs, lens, first, max_len, out, os, lse, w, ws, wb, None)


def _prefill(L, cache, attn, n=2, q=FAKE, qs=256, start=FAKE, lens=FAKE, max_len=64, out=FAKE, os=256, ws=FAKE, wb=1 << 30):
    return L.tman_attn_prefill(cache, attn, n, q, qs, start, lens, None, None, max_len, out, os, None, ws, wb, None)


def _evict(L, cache, w=FAKE, lens=FAKE, keep=16, recent=4, max_len=64, table=FAKE, pages=1, new=FAKE, kept=FAKE):
    return L.tman_kv_evict(cache, w, lens, keep, recent, max_len, table, pages, new, kept, None)


@pytest.mark.parametrize("over,status", [
    (dict(type=2), CACHE), (dict(type=-1), CACHE), (dict(dim=96), CACHE), (dict(dim=0), CACHE), (dict(dim=512), CACHE),
    (dict(page=8), CACHE), (dict(page=48), CACHE), (dict(page=2048), CACHE), (dict(page=0), CACHE), (dict(page=-16), CACHE),
    (dict(n_pages=0), SHAPE), (dict(n_seqs=0), SHAPE), (dict(n_seqs=65536), SHAPE), (dict(max_pages=0), SHAPE),
    (dict(max_pages=1 << 27), SHAPE), (dict(kv_heads=0), SHAPE),
    (dict(k_pages=None), NULL), (dict(v_pages=None), NULL), (dict(page_table=None), NULL),
    (dict(k_pages=FAKE + 8), ALIGN), (dict(v_pages=FAKE + 2), ALIGN),
])
def test_bad_caches_are_refused_everywhere(over, status):
    L, c, a = at._load(), _cache(**over), _attn()
    assert _append(L, c) == status
    assert _decode(L, c, a) == status
    assert _prefill(L, c, a) == status
    assert _evict(L, c) == status
    if status in (CACHE, SHAPE):
        assert L.tman_attn_decode_workspace_bytes(c, a, 64, 0) == 0
        assert L.tman_attn_prefill_workspace_bytes(c, a, 2, 64) == 0


def test_null_cache_and_attn():
    L, c, a = at._load(), _cache(), _attn()
    assert _append(L, None) == NULL and _decode(L, None, a) == NULL and _prefill(L, None, a) == NULL and _evict(L, None) == NULL
    assert _decode(L, c, None) == NULL and _prefill(L, c, None) == NULL


@pytest.mark.parametrize("attn", [_attn(heads=0), _attn(heads=3), _attn(heads=-2), _attn(heads=1 << 20), _attn(window=-1), _attn(cap=-1.0),
                                  _attn(scale=float("nan")), _attn(scale=float("inf")), _attn(cap=float("inf")),
                                  _attn(cap=float("nan"))])
def test_bad_score_rules(attn):
    L, c = at._load(), _cache()
    assert _decode(L, c, attn) == SHAPE and _prefill(L, c, attn) == SHAPE
    assert L.tman_attn_decode_workspace_bytes(c, attn, 64, 0) == 0


def test_bad_arguments():
    L, c, a = at._load(), _cache(), _attn()
    # rows: null, stride shorter than the heads, not a multiple of 8 elements, not aligned
    for call in (lambda **k: _decode(L, c, a, **k), lambda **k: _prefill(L, c, a, **k)):
        assert call(q=None) == NULL and call(out=None) == NULL and call(lens=None) == NULL
        assert call(qs=255) == SHAPE and call(os=248) == SHAPE
        assert call(qs=260) == ALIGN and call(os=257) == ALIGN and call(q=FAKE + 8) == ALIGN and call(out=FAKE + 2) == ALIGN
        assert call(max_len=0) == SHAPE and call(max_len=(1 << 30) + 1) == SHAPE
    need = L.tman_attn_decode_workspace_bytes(c, a, 64, 0)
    assert need > 0
    assert _decode(L, c, a, ws=None, wb=0) == WORKSPACE and _decode(L, c, a, wb=need - 1) == WORKSPACE
    assert _decode(L, c, a, ws=FAKE + 4, wb=need) == ALIGN and _decode(L, c, a, w=FAKE + 4) == ALIGN
    more = L.tman_attn_decode_workspace_bytes(c, a, 64, 1)
    assert more > need and _decode(L, c, a, w=FAKE, wb=need) == WORKSPACE
    assert _prefill(L, c, a, n=0) == SHAPE and _prefill(L, c, a, start=None) == NULL
    need = L.tman_attn_prefill_workspace_bytes(c, a, 2, 4096)
    assert need > 0 and _prefill(L, c, a, max_len=4096, ws=None, wb=0) == WORKSPACE
    assert _prefill(L, c, a, max_len=4096, wb=need - 1) == WORKSPACE
    assert L.tman_attn_prefill_workspace_bytes(c, a, 0, 64) == 0


def test_bad_append_arguments():
    L, c = at._load(), _cache()
    assert _append(L, c, n=0, start=FAKE) == SHAPE and _append(L, c, n=3) == SHAPE  # one token a sequence without q_start
    assert _append(L, c, q=None) == NULL and _append(L, c, qo=None) == NULL and _append(L, c, lens=None) == NULL
    assert _append(L, c, k=None) == NULL and _append(L, c, v=None) == NULL
    assert _append(L, c, heads=3) == SHAPE and _append(L, c, heads=0) == SHAPE
    assert _append(L, c, qs=128) == SHAPE and _append(L, c, qos=128) == SHAPE and _append(L, c, kvs=64) == SHAPE
    assert _append(L, c, qs=260) == ALIGN and _append(L, c, kvs=132) == ALIGN and _append(L, c, k=FAKE + 8) == ALIGN
    assert _append(L, c, v=FAKE + 8) == ALIGN and _append(L, c, qo=FAKE + 8) == ALIGN and _append(L, c, w=FAKE + 4) == ALIGN
    assert _append(L, c, pos=FAKE) == SHAPE  # positions without a table of angles
    for rope in (_rope(rot=0), _rope(rot=8), _rope(rot=24, sections=(12, 0, 0)), _rope(rot=128, sections=(64, 0, 0)),
                 _rope(n_pos=0), _rope(axes=0), _rope(axes=4), _rope(sections=(31, 0, 0)), _rope(interleaved=2),
                 _rope(axes=3, sections=(16, 32, -16)), _rope(axes=2, sections=(16, 15, 1))):
        assert _append(L, c, rope=rope) == SHAPE
    assert _append(L, c, rope=_rope(cos_sin=None)) == NULL and _append(L, c, rope=_rope(cos_sin=FAKE + 8)) == ALIGN


def test_bad_evict_arguments():
    L, c = at._load(), _cache()
    for name in ("w", "lens", "table", "new", "kept"):
        assert _evict(L, c, **{name: None}) == NULL
    assert _evict(L, c, keep=0) == SHAPE and _evict(L, c, recent=-1) == SHAPE and _evict(L, c, recent=17) == SHAPE
    assert _evict(L, c, max_len=0) == SHAPE and _evict(L, c, pages=0) == SHAPE and _evict(L, c, keep=17) == SHAPE  # one page of 16
    assert _evict(L, c, w=FAKE + 4) == ALIGN


def test_a_workspace_for_a_longer_bound_serves_shorter_ones():
    L = at._load()
    for kv_heads, heads, seqs in ((1, 1, 1), (8, 32, 1), (8, 32, 7), (5, 20, 3), (2, 40, 64), (32, 32, 300)):
        c = _cache(kv_heads=kv_heads, n_seqs=seqs, max_pages=1 << 20)
        for window in (0, 100, 5000):
            a = _attn(heads=heads, window=window)
            for weights in (0, 1):
                need = [L.tman_attn_decode_workspace_bytes(c, a, n, weights) for n in (1, 31, 33, 500, 1000, 1025, 4097, 40000, 131072)]
                assert need[0] >= 4096 * 4 and need == sorted(need)
            need = [L.tman_attn_prefill_workspace_bytes(c, a, 5, n) for n in (64, 257, 5000, 131072)]
            assert need == sorted(need)


def test_binding_refuses_tensors_that_do_not_fit():
    k = torch.zeros(8, 2, 16, 64, dtype=torch.float16)
    table = torch.zeros(2, 4, dtype=torch.int32)
    cache = tman.KvCache(k, k.clone(), table)
    attn = tman.Attn(4, 0.125)
    lens = torch.zeros(2, dtype=torch.int32)
    q, ws = torch.zeros(2, 4, 64, dtype=torch.float16), torch.zeros(1 << 20, dtype=torch.uint8)

    def status(f):
        with pytest.raises(tman.TmanError) as e:
            f()
        return e.value.status

    assert status(lambda: tman.KvCache(k.float(), k.float(), table)) == CACHE
    assert status(lambda: tman.KvCache(k, k.bfloat16(), table)) == CACHE
    assert status(lambda: tman.KvCache(k, k[:4], table)) == SHAPE
    assert status(lambda: tman.KvCache(k.transpose(1, 2), k.transpose(1, 2), table)) == SHAPE
    assert status(lambda: tman.KvCache(k, k, table.long())) == SHAPE
    assert status(lambda: tman.KvCache(k, k, table.t())) == SHAPE
    assert status(lambda: tman.Rope(torch.zeros(4, 32, 2, dtype=torch.float64))) == SHAPE
    assert status(lambda: tman.Rope(torch.zeros(4, 32, 2), (8, 8, 8, 8))) == SHAPE
    assert status(lambda: tman.Attn(4, 1.0, slopes=torch.zeros(3))) == SHAPE
    decode = lambda **over: tman.tman_attn_decode(  # noqa: E731
        cache, attn, **{**dict(q=q, lens=lens, out=q.clone(), max_len=64, workspace=ws, stream=0), **over})
    assert status(lambda: decode(q=q.bfloat16())) == CACHE
    assert status(lambda: decode(q=q[:1])) == SHAPE
    assert status(lambda: decode(q=q[:, :2])) == SHAPE
    assert status(lambda: decode(q=q.transpose(1, 2).contiguous().transpose(1, 2))) == SHAPE
    assert status(lambda: decode(q=None)) == NULL
    assert status(lambda: decode(lens=lens.long())) == SHAPE
    assert status(lambda: decode(lens=lens[:1])) == SHAPE
    assert status(lambda: decode(lens=None)) == NULL
    assert status(lambda: decode(first=lens[:1])) == SHAPE
    assert status(lambda: decode(lse=torch.zeros(2, 3))) == SHAPE
    assert status(lambda: decode(weights=torch.zeros(8, 2, 8))) == SHAPE
    assert status(lambda: decode(workspace=None)) == WORKSPACE
    prefill = lambda **over: tman.tman_attn_prefill(  # noqa: E731
        cache, attn, **{**dict(q=q, q_start=torch.zeros(3, dtype=torch.int32), lens=lens, out=q.clone(), max_len=64, workspace=ws,
                               stream=0), **over})
    assert status(lambda: prefill(q_start=lens)) == SHAPE
    assert status(lambda: prefill(first=torch.zeros(3, dtype=torch.int32))) == SHAPE
    assert status(lambda: prefill(end=torch.zeros(2))) == SHAPE
    kv = torch.zeros(2, 2, 64, dtype=torch.float16)
    append = lambda **over: tman.tman_rope_append(  # noqa: E731
        cache, **{**dict(q=q, k=kv, v=kv, lens=lens, q_out=q, stream=0), **over})
    assert status(lambda: append(k=kv[:, :1])) == SHAPE
    assert status(lambda: append(v=torch.zeros(2, 2, 128, dtype=torch.float16)[..., :64])) == SHAPE
    assert status(lambda: append(q_out=None)) == NULL
    assert status(lambda: append(positions=lens)) == SHAPE
    evict = lambda **over: tman.tman_kv_evict(  # noqa: E731
        cache, **{**dict(weights=torch.zeros(8, 2, 16), lens=lens, keep=16, recent=0, new_table=torch.zeros(2, 1, dtype=torch.int32),
                         new_lens=lens, kept=torch.zeros(2, 2, 16, dtype=torch.int32), max_len=64, stream=0), **over})
    assert status(lambda: evict(kept=torch.zeros(2, 2, 15, dtype=torch.int32))) == SHAPE
    assert status(lambda: evict(weights=None)) == NULL
    assert status(lambda: evict(new_table=torch.zeros(3, 1, dtype=torch.int32))) == SHAPE


def test_rows_are_numbered_in_32_bits():
    L, c, a = at._load(), _cache(n_seqs=65535, kv_heads=2), _attn(heads=65536)
    assert _decode(L, c, a, qs=1 << 23, os=1 << 23) == SHAPE and L.tman_attn_decode_workspace_bytes(c, a, 64, 0) == 0
    assert _prefill(L, c, a, n=40000, qs=1 << 23, os=1 << 23) == SHAPE and L.tman_attn_prefill_workspace_bytes(c, a, 40000, 64) == 0
    assert _append(L, c, n=(1 << 30) + 1, start=FAKE) == SHAPE


def test_status_strings():
    assert len({tman.tman_status_string(c) for c in range(0, -11, -1)}) == 11
