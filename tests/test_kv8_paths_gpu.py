"""Paths of the 8-bit cache's operators that only large calls take, what a used workspace may hold, and what exactly is finite at the ends of
the types."""
import pytest
import torch

import kv8_ref as ref
import paper_2511_11248_amd as tman
from attention_ref import attend
from gpu_helpers import dev
from test_kv8_append_gpu import Cache8, angles, check
from test_kv8_attention_gpu import Problem8, check_decode, check_prefill, mask_of, within

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
TICKETS = 16384  # bytes in front of a workspace that a caller zeroes; the rest is what the calls before have left


def sane(C):
    """Older positions as codes of finite values, exponents of about one."""
    for b, n in enumerate(C.lens_list):
        used = C.table[b, :-(-n // C.page)].long()
        for pages, exps in ((C.k, C.ke), (C.v, C.ve)):
            pages[used] = (C.normal(len(used), *pages.shape[1:]) * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            exps[used] = 119 + b % 4


def heads_a_wave(kv_heads, items):
    """Of a block, as the launch shares them out: a wave keeps angles and shared weights over them, and has the next one's rows on their way."""
    return min(max(1, (kv_heads * 2 * items + 1024) // 2048), kv_heads)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("weights", ["none", "shared", "per head"])
@pytest.mark.parametrize("lens,new,kv_heads", [([1100, 45], [1100, 30], 24), ([700, 650, 90], [690, 513, 1], 40)])
def test_appends_whose_waves_take_several_heads(dim, weights, lens, new, kv_heads):
    assert heads_a_wave(kv_heads, (sum(new) + 30 * len(new)) // 16) > 1
    C = Cache8(dim + kv_heads, lens, kv_heads, kv_heads, dim, 32, torch.bfloat16 if dim == 128 else torch.float16)
    sane(C)
    norm = None
    if weights != "none":
        shape = (kv_heads, dim) if weights == "per head" else (dim,)
        norm = tman.HeadNorm(1 + 0.3 * C.normal(*shape), 1 + 0.3 * C.normal(*shape), 1e-6)
    check(C, new, rule=(angles(1200, dim // 2), (dim // 4,), dim == 128), norm=norm, magnitude=2.0, q=weights != "none")


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("normed", [False, True])
def test_single_tokens_whose_waves_take_several_heads(dim, normed):
    lens = [(13 * b * b) % 70 + 1 for b in range(96)]
    C = Cache8(dim, lens, 32, 32, dim, 16, torch.float16)
    assert heads_a_wave(32, len(lens)) == 3
    sane(C)
    norm = tman.HeadNorm(None, 1 + 0.3 * C.normal(32, dim), 1e-6) if normed else None
    check(C, [1] * 96, rule=(angles(80, dim), (dim // 2,), False), norm=norm, starts=False, magnitude=8.0)


@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 4, 1), (128, 6, 2), (256, 4, 1)])
@pytest.mark.parametrize("how", [dict(), dict(window=70), dict(mask="documents"), dict(mask="prefix", sloped=True), dict(cap=30.0)])
def test_prompts_whose_copy_would_not_fit(dim, heads, kv_heads, how):
    """A bound of half a milliard positions: codes are read for every 32 rows."""
    how = dict(how)
    lens, new = [700, 333], [190, 333]
    first, end = mask_of(how.pop("mask", "causal"), lens, new)
    P = Problem8(dim, lens, heads, kv_heads, dim, 32, torch.float16)
    bound = 1 << 29
    assert 4 * 2 * bound * kv_heads * dim > 16 << 30
    attn = tman.Attn(heads, 1.0)
    need = tman.tman_attn_prefill_kv8_workspace_bytes(P.cache, attn, sum(new) + 3, bound)
    plan = 64 << 20  # what the call itself needs is far below the room for every shorter bound
    ws = torch.full((plan,), 0xff, dtype=torch.uint8, device=dev())
    ws[:TICKETS] = 0
    assert need > plan
    check_prefill(P, new, first, end, workspace=ws, bound_len=bound, sample=[0, 50, 100, 188, 300], **how)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 1024), (256, 32)])
@pytest.mark.parametrize("how", [dict(), dict(window=1), dict(window=63), dict(window=500), dict(mask="documents"), dict(mask="prefix"),
                                 dict(mask="empty"), dict(sloped=True, window=100), dict(cap=20.0)])
@pytest.mark.parametrize("many", [False, True])
def test_what_a_workspace_holds_does_not_matter(dtype, dim, page, how, many):
    """Everything behind the tickets is NaN in both types: places that the copy leaves out are never read."""
    how = dict(how)
    lens, new = ([2101, 0, 333, 1999], [1101, 0, 333, 700]) if many else ([301, 33, 700], [5, 33, 9])
    first, end = mask_of(how.pop("mask", "causal"), lens, new)
    P = Problem8(dim + page, lens, 4, 1, dim, page, dtype)
    for bound in (max(lens), 2600):
        ws = torch.full((128 << 20,), 0xff, dtype=torch.uint8, device=dev())
        ws[:TICKETS] = 0
        check_prefill(P, new, first, end, workspace=ws, bound_len=bound, sample=[0, 62, 63, 64, 500, 698], **how)
        assert not bool(ws[:TICKETS].any())
        check_decode(P, workspace=ws, bound_len=bound, **{k: v for k, v in how.items()})


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("many", [False, True])
def test_blocks_of_overflowing_values_that_some_rows_must_not_see(dim, many):
    """A block whose exponent takes its keys and values out of fp16: rows ahead of it are as if it were not there."""
    lens, new = ([2500], [900]) if many else ([300], [40])
    P = Problem8(43, lens, 4, 1, dim, 16, torch.float16)
    n, t = lens[0], new[0]
    block = (n - t // 2) // 16 * 16
    page, _ = P.row(0, block)
    P.ve[page], P.ke[page] = 200, 200
    P.v[page] |= 0x40  # (codes of two and more: infinities all)
    P.v[page] = torch.where((P.v[page] & 0x7f) == 0x7f, 0x48, P.v[page])
    H, scale = 4, dim ** -0.5
    q = P.normal(t, H, dim)
    out, lse = torch.empty_like(q), torch.empty(t, H, device=dev())
    attn = tman.Attn(H, scale)
    ws = torch.zeros(max(16, tman.tman_attn_prefill_kv8_workspace_bytes(P.cache, attn, t, n)), dtype=torch.uint8, device=dev())
    tman.tman_attn_prefill_kv8(P.cache, attn, q, P.ints([0, t]), P.lens, out, n, ws, lse=lse)
    assert tman.tman_device_status() == 0
    sees = torch.arange(n - t, n, device=dev()) >= block
    assert bool(torch.isfinite(out[~sees]).all()) and bool(torch.isfinite(lse[~sees]).all())
    assert not bool(torch.isfinite(out[sees]).any())
    k, v = P.rows(P.k, P.ke, 0, block), P.rows(P.v, P.ve, 0, block)
    for i in (0, t // 4, block - (n - t) - 1):
        at = n - t + i
        o, l, _, bound, l_bound, _ = attend(q[i], k, v, at, 0, at + 1, scale, 0.0, None, 0, torch.float16)
        within(out[i], o, bound, f"out of token {i}")
        within(lse[i], l, l_bound, f"lse of token {i}")


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_what_is_finite_at_the_ends_of_the_types(dtype, dim):
    """Every place by itself: NaN where an infinity or NaN was written, a number of the type anywhere else, also beside them."""
    top, C = torch.finfo(dtype).max, Cache8(5, [96], 2, 2, dim, 32, dtype)
    kv = (C.normal(96, 4, dim) * 3).to(dtype)
    want = torch.ones(96, dim, dtype=torch.bool, device=dev())
    for j, d, x in ((16, 3, top), (17, 4, -top), (32, 5, INF), (33, 6, NAN), (34, 7, -INF), (40, dim - 1, INF), (64, 0, top * 0.875), (65, 1, -top * 0.9)):
        kv[j, :, d] = x
        want[j, d] = abs(x) <= top
    kv[48:64], want[48:64] = INF, False
    kv[80:96, :, 1] = top
    kv[81, :, 2], want[81, 2] = NAN, False
    tman.tman_kv8_append(C.cache, None, kv[:, :2], kv[:, 2:], C.lens, None, q_start=C.ints([0, 96]))
    assert tman.tman_device_status() == 0
    for pages, exps in ((C.k, C.ke), (C.v, C.ve)):
        for h in range(2):
            x = ref.decode(C.head(pages, 0, h, 96)[None], C.head(exps, 0, h, 96)[None])[0]
            assert torch.equal(torch.isfinite(x.to(dtype)), want)
            assert torch.equal(torch.isnan(x), ~want)
