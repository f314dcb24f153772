"""Host-side checks of the operators around a cache held in 8 bits and of the pages of a step: size queries, and refusals before
anything is launched."""
import ctypes as C
import gc
import weakref

import pytest
import torch

import paper_2511_11248_amd as tman
from paper_2511_11248_amd import attention as at

FAKE = 0x1000  # non-NULL, 16-byte aligned, never dereferenced: validation fails first
NULL, SHAPE, WORKSPACE, ALIGN, CACHE = -1, -4, -5, -6, -9


def _cache(ke=FAKE, ve=FAKE, **over):
    f = dict(k_pages=FAKE, v_pages=FAKE, page_table=FAKE, n_pages=8, n_seqs=2, max_pages=4, kv_heads=2, page=16, dim=64, type=0)
    f.update(over)
    return C.byref(at._CCache8(at._CCache(*[f[n] for n, _ in at._CCache._fields_]), ke, ve))


def _attn(heads=4, window=0, scale=1.0, cap=0.0, slopes=None):
    return C.byref(at._CAttn(heads, window, scale, cap, slopes))


def _norm(q=FAKE, k=FAKE, eps=1e-6, per_head=0):
    return C.byref(at._CNorm(q, k, eps, per_head))


def _append(L, cache, norm=None, rope=None, heads=4, n=2, q=FAKE, qs=256, k=FAKE, v=FAKE, kvs=128, pos=None, start=None, lens=FAKE,
            qo=FAKE, qos=256):
    return L.tman_kv8_append(cache, norm, rope, heads, n, q, qs, k, v, kvs, pos, start, lens, qo, qos, None)


def _decode(L, cache, attn, q=FAKE, qs=256, lens=FAKE, max_len=64, out=FAKE, os=256, ws=FAKE, wb=1 << 30):
    return L.tman_attn_decode_kv8(cache, attn, q, qs, lens, None, max_len, out, os, None, ws, wb, None)


def _prefill(L, cache, attn, n=2, q=FAKE, qs=256, start=FAKE, lens=FAKE, max_len=64, out=FAKE, os=256, ws=FAKE, wb=1 << 30):
    return L.tman_attn_prefill_kv8(cache, attn, n, q, qs, start, lens, None, None, max_len, out, os, None, ws, wb, None)


@pytest.mark.parametrize("over,status", [
    (dict(type=2), CACHE), (dict(dim=96), CACHE), (dict(dim=512), CACHE), (dict(page=8), CACHE), (dict(page=48), CACHE),
    (dict(page=2048), CACHE), (dict(n_pages=0), SHAPE), (dict(n_seqs=0), SHAPE), (dict(n_seqs=65536), SHAPE), (dict(max_pages=0), SHAPE),
    (dict(max_pages=1 << 27), SHAPE), (dict(kv_heads=0), SHAPE), (dict(n_pages=2 ** 31 - 1, kv_heads=4096), SHAPE),
    (dict(k_pages=None), NULL), (dict(v_pages=None), NULL), (dict(page_table=None), NULL), (dict(ke=None), NULL), (dict(ve=None), NULL),
    (dict(k_pages=FAKE + 8), ALIGN), (dict(v_pages=FAKE + 2), ALIGN), (dict(ke=FAKE + 1), ALIGN), (dict(ve=FAKE + 2), ALIGN),
])
def test_bad_caches_are_refused_everywhere(over, status):
    L, c, a = at._load(), _cache(**over), _attn()
    assert _append(L, c) == status and _decode(L, c, a) == status and _prefill(L, c, a) == status
    if status in (CACHE, SHAPE):
        assert L.tman_attn_decode_kv8_workspace_bytes(c, a, 64) == 0
        assert L.tman_attn_prefill_kv8_workspace_bytes(c, a, 2, 64) == 0


def test_bad_arguments():
    L, c, a = at._load(), _cache(), _attn()
    assert _append(L, None) == NULL and _decode(L, None, a) == NULL and _prefill(L, None, a) == NULL
    assert _decode(L, c, None) == NULL and _prefill(L, c, None) == NULL
    for attn in (_attn(heads=0), _attn(heads=3), _attn(window=-1), _attn(cap=-1.0), _attn(scale=float("nan"))):
        assert _decode(L, c, attn) == SHAPE and _prefill(L, c, attn) == SHAPE
    assert _append(L, c, n=0) == SHAPE and _append(L, c, n=3) == SHAPE and _append(L, c, heads=3) == SHAPE
    assert _append(L, c, k=None) == NULL and _append(L, c, v=None) == NULL and _append(L, c, lens=None) == NULL
    assert _append(L, c, qo=None) == NULL and _append(L, c, q=None) == NULL
    assert _append(L, c, kvs=120) == SHAPE and _append(L, c, qs=260) == ALIGN and _append(L, c, k=FAKE + 2) == ALIGN
    assert _append(L, c, pos=FAKE) == SHAPE  # positions without a rotation
    assert _decode(L, c, a, lens=None) == NULL and _decode(L, c, a, q=None) == NULL and _decode(L, c, a, out=None) == NULL
    assert _decode(L, c, a, max_len=0) == SHAPE and _decode(L, c, a, os=8) == SHAPE
    assert _decode(L, c, a, ws=None) == WORKSPACE and _decode(L, c, a, wb=8) == WORKSPACE and _decode(L, c, a, ws=FAKE + 8) == ALIGN
    assert _prefill(L, c, a, start=None) == NULL and _prefill(L, c, a, n=0) == SHAPE and _prefill(L, c, a, n=2 ** 31 - 1) == SHAPE


@pytest.mark.parametrize("norm,status", [(dict(eps=0.0), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE),
                                         (dict(eps=float("inf")), SHAPE), (dict(eps=1e-31), SHAPE), (dict(per_head=2), SHAPE),
                                         (dict(q=FAKE + 4), ALIGN), (dict(k=FAKE + 8), ALIGN)])
def test_bad_norms(norm, status):
    L = at._load()
    assert _append(L, _cache(), norm=_norm(**norm)) == status
    c16 = C.byref(at._CCache(FAKE, FAKE, FAKE, 8, 2, 4, 2, 16, 64, 0))
    args = (None, 4, 2, FAKE, 256, FAKE, FAKE, 128, None, None, FAKE, FAKE, 256, None, None)
    assert L.tman_norm_rope_append(c16, _norm(**norm), *args) == status
    assert L.tman_norm_rope_append(c16, None, *args) == NULL


def test_workspaces():
    L, a = at._load(), _attn()
    c = _cache(n_pages=1 << 20, max_pages=1 << 20, page=16)
    decode = [L.tman_attn_decode_kv8_workspace_bytes(c, a, n) for n in (1, 100, 10000, 1 << 20)]
    assert decode == sorted(decode) and decode[0] > 0
    # a longer bound never needs less, also where the copy of a prompt's values no longer fits and there is none
    bounds = [1, 64, 2048, 2049, 5000, 1 << 16, 1 << 20, 1 << 23]
    prefill = [L.tman_attn_prefill_kv8_workspace_bytes(c, a, 4096, n) for n in bounds]
    assert prefill == sorted(prefill)
    values = 2 * 2 * 5008 * 2 * 64 * 2
    assert values <= prefill[4] < values + (64 << 20)  # (with the pieces of rows)
    assert (16 << 30) - (64 << 20) <= L.tman_attn_prefill_kv8_workspace_bytes(_cache(n_seqs=1, n_pages=1 << 20, max_pages=1 << 16, page=1024, kv_heads=16, dim=256),
                                                                         _attn(heads=16), 4096, 1 << 26) < (16 << 30) + (64 << 20)
    assert _prefill(L, c, a, n=4096, max_len=5000, wb=values) == WORKSPACE


def _plan(L, table=FAKE, B=2, pages=4, page=16, lens=FAKE, more=0x2000, stack=0x3000, cap=8, left=0x4000, n=16, new=0x5000, new_left=0x6000,
          start=0x7000, slots=None, pos=None, own=None, ws=None, wb=0):
    return L.tman_kv_plan(table, B, pages, page, lens, more, stack, cap, left, n, new, new_left, start, slots, pos, own, ws, wb, None)


@pytest.mark.parametrize("over,status", [
    (dict(table=None), NULL), (dict(lens=None), NULL), (dict(more=None), NULL), (dict(stack=None), NULL), (dict(left=None), NULL),
    (dict(new=None), NULL), (dict(new_left=None), NULL), (dict(start=None), NULL), (dict(page=8), CACHE), (dict(page=24), CACHE),
    (dict(page=2048), CACHE), (dict(B=0), SHAPE), (dict(B=65536), SHAPE), (dict(pages=0), SHAPE), (dict(pages=1 << 27), SHAPE),
    (dict(cap=0), SHAPE), (dict(n=0), SHAPE), (dict(n=(1 << 30) + 1), SHAPE), (dict(new=FAKE + 4), SHAPE), (dict(slots=FAKE + 4), ALIGN),
    (dict(n=1 << 20), WORKSPACE), (dict(n=1 << 20, ws=FAKE, wb=4), WORKSPACE), (dict(n=1 << 20, ws=FAKE + 4, wb=1 << 10), ALIGN),
])
def test_bad_plans(over, status):
    assert _plan(at._load(), **over) == status


def test_plan_workspaces():
    size = tman.tman_kv_plan_workspace_bytes
    assert size(8, 8) == 0 and size(8, 1 << 20) >= 32 and size(0, 8) == 0 and size(8, 0) == 0 and size(65536, 8) == 0


def _tensors(B=2, H=4, G=2, D=64, page=16):
    pages = torch.zeros(8, G, page, D, dtype=torch.uint8).view(torch.float8_e4m3fn)
    exps = torch.zeros(8, G, page // 16, dtype=torch.uint8)
    rows = {name: torch.zeros(B, n, D, dtype=torch.float16) for name, n in (("q", H), ("k", G), ("v", G), ("out", H))}
    return dict(k_pages=pages, v_pages=pages.clone(), k_exps=exps, v_exps=exps.clone(), table=torch.zeros(B, 4, dtype=torch.int32), **rows,
                lens=torch.zeros(B, dtype=torch.int32), q_start=torch.arange(B + 1, dtype=torch.int32), q_weight=torch.ones(D), k_weight=torch.ones(D),
                cos_sin=torch.zeros(8, D // 2, 2), first=torch.zeros(B, dtype=torch.int32), lse=torch.zeros(B, H),
                workspace=torch.zeros(1 << 20, dtype=torch.uint8))


def _handle(t, dtype=torch.float16):
    return tman.KvCache8(t["k_pages"], t["v_pages"], t["k_exps"], t["v_exps"], t["table"], dtype)


@pytest.mark.parametrize("bad", [dict(k_exps=torch.zeros(8, 2, 2, dtype=torch.uint8)), dict(v_exps=torch.zeros(8, 2, 1)),
                                 dict(v_pages=torch.zeros(8, 2, 16, 64, dtype=torch.float16)), dict(table=torch.zeros(8, dtype=torch.int32)),
                                 dict(k_pages=torch.zeros(7, 2, 16, 64, dtype=torch.uint8))])
def test_tensors_that_are_no_cache(bad):
    with pytest.raises(tman.TmanError):
        _handle({**_tensors(), **bad})


def test_handles_of_the_other_kind_are_refused():
    t = _tensors()
    c8 = _handle(t)
    half = torch.zeros(8, 2, 16, 64, dtype=torch.float16)
    c16 = tman.KvCache(half, half.clone(), t["table"])
    attn = tman.Attn(4, 1.0)
    for call in (lambda: tman.tman_rope_append(c8, t["q"], t["k"], t["v"], t["lens"], t["out"]),
                 lambda: tman.bound_rope_append(c8, t["q"], t["k"], t["v"], t["lens"], t["out"]),
                 lambda: tman.tman_norm_rope_append(c8, tman.HeadNorm(None, None, 1e-6), t["q"], t["k"], t["v"], t["lens"], t["out"]),
                 lambda: tman.tman_kv8_append(c16, t["q"], t["k"], t["v"], t["lens"], t["out"]),
                 lambda: tman.tman_attn_decode(c8, attn, t["q"], t["lens"], t["out"], 64, t["workspace"]),
                 lambda: tman.bound_attn_decode(c8, attn, t["q"], t["lens"], t["out"], 64, t["workspace"]),
                 lambda: tman.tman_attn_decode_kv8(c16, attn, t["q"], t["lens"], t["out"], 64, t["workspace"]),
                 lambda: tman.tman_attn_prefill(c8, attn, t["q"], t["q_start"], t["lens"], t["out"], 64, t["workspace"]),
                 lambda: tman.tman_attn_prefill_kv8(c16, attn, t["q"], t["q_start"], t["lens"], t["out"], 64, t["workspace"]),
                 lambda: tman.tman_kv_evict(c8, torch.zeros(8, 2, 16), t["lens"], 16, 4, t["table"], t["lens"], t["lens"], 64),
                 lambda: tman.tman_attn_decode_workspace_bytes(c8, attn, 64),
                 lambda: tman.tman_attn_prefill_kv8_workspace_bytes(c16, attn, 4, 64)):
        with pytest.raises(tman.TmanError) as e:
            call()
        assert e.value.status == CACHE


def test_norm_weights_fit_their_heads():
    t = _tensors()
    c8 = _handle(t)
    for q, k in ((torch.ones(32), torch.ones(64)), (torch.ones(4, 64), torch.ones(4, 64)), (torch.ones(2, 64), torch.ones(2, 64))):
        with pytest.raises(tman.TmanError):
            tman.tman_kv8_append(c8, t["q"], t["k"], t["v"], t["lens"], t["out"], norm=tman.HeadNorm(q, k, 1e-6))
    with pytest.raises(tman.TmanError):
        tman.HeadNorm(torch.ones(64), torch.ones(2, 64), 1e-6)
    with pytest.raises(tman.TmanError):
        tman.HeadNorm(torch.ones(64).half(), None, 1e-6)
    with pytest.raises(tman.TmanError):
        tman.tman_norm_rope_append(c8, None, t["q"], t["k"], t["v"], t["lens"], t["out"])


@pytest.mark.parametrize("bind,used", [
    (lambda t: tman.bound_kv8_append(_handle(t), t["q"], t["k"], t["v"], t["lens"], t["out"], norm=tman.HeadNorm(t["q_weight"], t["k_weight"], 1e-6),
                                     rope=tman.Rope(t["cos_sin"]), q_start=t["q_start"]),
     "k_pages v_pages k_exps v_exps table q k v lens out q_weight k_weight cos_sin q_start"),
    (lambda t: tman.bound_attn_decode_kv8(_handle(t), tman.Attn(4, 1.0), t["q"], t["lens"], t["out"], 64, t["workspace"], first=t["first"],
                                          lse=t["lse"]), "k_pages v_pages k_exps v_exps table q lens out workspace first lse"),
])
def test_a_bound_call_keeps_its_tensors(bind, used):
    t = _tensors()
    call = bind(t)
    alive = {name: weakref.ref(t[name]) for name in used.split()}
    del t
    gc.collect()
    assert [name for name, ref in alive.items() if ref() is None] == []
    del call
    gc.collect()
    assert [name for name, ref in alive.items() if ref() is not None] == []


def _plan_tensors(B=3, pages=4, n=8):
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    return dict(page_table=ints(B, pages), page=16, lens=ints(B), more=ints(B), free_pages=ints(9), free_left=ints(1), new_lens=ints(B),
                new_left=ints(1), q_start=ints(B + 1), slots=torch.zeros(n, dtype=torch.int64), positions=ints(n), owners=ints(n))


@pytest.mark.parametrize("name,bad,status", [
    *((n, None, NULL) for n in ("page_table", "lens", "more", "free_pages", "free_left", "new_lens", "new_left", "q_start")),
    *((n, torch.zeros(3), SHAPE) for n in ("lens", "more", "free_pages", "free_left", "new_lens", "new_left", "q_start", "slots", "positions", "owners")),
    ("page_table", torch.zeros(3, 4), SHAPE), ("page_table", torch.zeros(12, dtype=torch.int32), SHAPE),
    ("lens", torch.zeros(4, dtype=torch.int32), SHAPE), ("q_start", torch.zeros(3, dtype=torch.int32), SHAPE),
    ("more", torch.zeros(6, dtype=torch.int32)[::2], SHAPE), ("q_start", torch.zeros(8, dtype=torch.int32)[::2], SHAPE),
    ("positions", torch.zeros(7, dtype=torch.int32), SHAPE), ("slots", torch.zeros(8, dtype=torch.int32), SHAPE), ("page", 24, CACHE),
])
def test_tensors_that_are_no_plan(name, bad, status):
    for call in (lambda **a: tman.tman_kv_plan(stream=0, **a), tman.bound_kv_plan):
        if call is tman.bound_kv_plan and name == "page":
            continue  # (the library's own checks come with the call)
        with pytest.raises(tman.TmanError) as e:
            call(**{**_plan_tensors(), name: bad})
        assert e.value.status == status
    with pytest.raises(tman.TmanError):
        tman.tman_kv_plan(stream=0, **{**_plan_tensors(), "slots": None, "positions": None, "owners": None})
