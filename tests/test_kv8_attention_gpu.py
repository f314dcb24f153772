"""Attention over a cache held in 8 bits against a plain 64-bit form of the values that the codes stand for: types, head sizes and
groups, pages, lengths from none to several pieces, masks, values that must not be seen, strides, workspaces, the copy of long prompts."""
import pytest
import torch

import kv8_ref as ref
import paper_2511_11248_amd as tman
from attention_ref import attend
from gpu_helpers import dev
from test_attention_gpu import within

pytestmark = pytest.mark.gpu
ERR_INDEX = -10
NAN = float("nan")


class Problem8:
    """Sequences in a cache of shuffled pages.  What lies behind a sequence's end is NaN codes, the exponents of blocks of nobody are
    255; table entries that are not used are no pages."""

    def __init__(self, seed, lens, heads, kv_heads, dim, page, dtype, extra=2):
        self.gen = torch.Generator(device=dev())
        self.gen.manual_seed(seed)
        self.lens_list, self.heads, self.kv_heads, self.dim, self.page, self.dtype = lens, heads, kv_heads, dim, page, dtype
        wide = max(1, max((n + page - 1) // page for n in lens)) + 1
        n_pages = sum((n + page - 1) // page for n in lens) + extra
        order = torch.randperm(n_pages, generator=self.gen, device=dev()).tolist()
        shape = (n_pages, kv_heads, page, dim)
        self.k, self.v = self.codes(*shape), self.codes(*shape)
        self.ke, self.ve = (torch.randint(117, 123, (*shape[:2], page // 16), generator=self.gen, device=dev(), dtype=torch.uint8)
                            for _ in range(2))
        own = torch.zeros(n_pages, page, dtype=torch.bool, device=dev())
        table = torch.full((len(lens), wide), 2 ** 30, dtype=torch.int32)
        for b, n in enumerate(lens):
            for i in range((n + page - 1) // page):
                table[b, i] = order.pop()
                own[table[b, i], :n - i * page] = True
        hidden = ~own[:, None, :, None].expand_as(self.k)
        self.k[hidden], self.v[hidden] = 0x7f, 0xff
        nobody = ~own.view(n_pages, page // 16, 16).any(-1)[:, None].expand_as(self.ke)
        self.ke[nobody], self.ve[nobody] = 255, 255
        self.table, self.lens = table.to(dev()), self.ints(lens)
        self.cache = tman.KvCache8(self.k, self.v, self.ke, self.ve, self.table, dtype)

    def codes(self, *shape):
        x = torch.randn(*shape, generator=self.gen, device=dev()) * 100
        return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.gen, device=dev()).to(self.dtype)

    def ints(self, x):
        return torch.tensor(x, dtype=torch.int32, device=dev())

    def slopes(self):
        return torch.tensor([2.0 ** (-8.0 * (h + 1) / self.heads) for h in range(self.heads)], dtype=torch.float32, device=dev())

    def rows(self, pages, exps, b, n):
        """[kv_heads, n, dim] of sequence b, in 64 bits."""
        used = self.table[b, :(n + self.page - 1) // self.page].long()
        x = ref.decode(pages[used], exps[used]).transpose(0, 1)
        return x.reshape(x.shape[0], -1, self.dim)[:, :n] if n else x.reshape(self.kv_heads, 0, self.dim)

    def row(self, b, j):
        return int(self.table[b, j // self.page]), j % self.page


def check_decode(P, first=None, cap=0.0, window=0, sloped=False, scale=None, workspace=None, bound_len=None):
    B, H, G, D = len(P.lens_list), P.heads, P.kv_heads, P.dim
    scale = D ** -0.5 if scale is None else scale
    q = P.normal(B, H + 2 * G, D)[:, :H]
    out = torch.full((B, H + 1, D), 7.0, dtype=P.dtype, device=dev())[:, :H]
    lse = torch.full((B, H), NAN, device=dev())
    slopes = P.slopes() if sloped else None
    attn = tman.Attn(H, scale, cap=cap, window=window, slopes=slopes)
    max_len = bound_len or max(1, max(P.lens_list))
    ws = workspace
    if ws is None:
        ws = torch.zeros(tman.tman_attn_decode_kv8_workspace_bytes(P.cache, attn, max_len), dtype=torch.uint8, device=dev())
    tman.tman_attn_decode_kv8(P.cache, attn, q, P.lens, out, max_len, ws, first=None if first is None else P.ints(first), lse=lse)
    assert tman.tman_device_status() == 0
    for b, n in enumerate(P.lens_list):
        lo = 0 if first is None else max(first[b], 0)
        o, l, _, bound, l_bound, _ = attend(q[b], P.rows(P.k, P.ke, b, n), P.rows(P.v, P.ve, b, n), n - 1, lo, n, scale, cap, slopes, window,
                                            P.dtype)
        within(out[b], o, bound, f"out[{b}], length {n}")
        within(lse[b], l, l_bound, f"lse[{b}], length {n}")
    return out, ws


def check_prefill(P, new, first=None, end=None, cap=0.0, window=0, sloped=False, scale=None, workspace=None, bound_len=None, sample=None):
    B, H, G, D = len(P.lens_list), P.heads, P.kv_heads, P.dim
    scale = D ** -0.5 if scale is None else scale
    N, spare = sum(new), 3
    q = P.normal(N + spare, H + 2 * G, D)[:, :H]
    out = torch.full((N + spare, H + 1, D), 7.0, dtype=P.dtype, device=dev())[:, :H]
    lse = torch.full((N + spare, H), 7.0, device=dev())
    slopes = P.slopes() if sloped else None
    attn = tman.Attn(H, scale, cap=cap, window=window, slopes=slopes)
    max_len = bound_len or max(1, max(P.lens_list))
    starts = [sum(new[:b]) for b in range(B + 1)]
    pad = lambda x: None if x is None else P.ints(list(x) + [0] * spare)  # noqa: E731
    ws = workspace
    if ws is None:
        need = tman.tman_attn_prefill_kv8_workspace_bytes(P.cache, attn, N + spare, max_len)
        ws = torch.zeros(need, dtype=torch.uint8, device=dev()) if need else None
    tman.tman_attn_prefill_kv8(P.cache, attn, q, P.ints(starts), P.lens, out, max_len, ws, first=pad(first), end=pad(end), lse=lse)
    assert tman.tman_device_status() == 0
    for b, (n, t) in enumerate(zip(P.lens_list, new)):
        k, v = P.rows(P.k, P.ke, b, n), P.rows(P.v, P.ve, b, n)
        for i in range(t) if sample is None else sorted({0, t - 1, *(x % t for x in sample)} if t else []):
            x, at = starts[b] + i, n - t + i
            lo = 0 if first is None else first[x]
            hi = min(n, at + 1 if end is None else end[x])
            o, l, _, bound, l_bound, _ = attend(q[x], k, v, at, lo, hi, scale, cap, slopes, window, P.dtype)
            within(out[x], o, bound, f"out of token {i} of sequence {b}")
            within(lse[x], l, l_bound, f"lse of token {i} of sequence {b}")
    assert bool((out[N:] == 7).all()) and bool((lse[N:] == 7).all())  # rows behind the last sequence
    return out, ws


LENS = [1, 0, 15, 16, 17, 31, 32, 33, 127, 128, 129, 300, 1027]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads,page", [(4, 4, 16), (6, 2, 32), (8, 1, 64), (20, 1, 128), (32, 2, 256), (5, 5, 1024)])
def test_decode_lengths(dtype, dim, heads, kv_heads, page):
    check_decode(Problem8(dim + heads, LENS, heads, kv_heads, dim, page, dtype))


@pytest.mark.parametrize("dtype,dim,page", [(torch.float16, 64, 16), (torch.bfloat16, 128, 32), (torch.float16, 256, 64)])
@pytest.mark.parametrize("rule", [dict(cap=20.0), dict(sloped=True), dict(cap=30.0, sloped=True), dict(window=1), dict(window=40),
                                  dict(window=333, cap=5.0), dict(window=5000), dict(scale=-0.3), dict(scale=0.0), dict(cap=1000.0)])
def test_decode_rules(dtype, dim, page, rule):
    check_decode(Problem8(3 + dim, [1, 0, 40, 41, 72, 500, 2049], 10, 2, dim, page, dtype), **rule)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_decode_first_hides_leading_positions_whatever_they_hold(dim):
    lens = [50, 50, 50, 50, 700, 700, 0, 3]
    first = [0, 7, 49, 50, 133, 900, 5, -4]  # also nothing left, beyond the end, before the start
    P = Problem8(11, lens, 8, 2, dim, 16, torch.float16)
    for b, (n, f) in enumerate(zip(lens, first)):
        for j in range(0, min(max(f, 0), n)):
            page, slot = P.row(b, j)
            P.k[page, :, slot], P.v[page, :, slot] = 0x7f, 0xff
            if j + 16 <= f and j % 16 == 0:
                P.ke[page], P.ve[page] = 255, 255
    out, _ = check_decode(P, first=first)
    assert bool((out[3] == 0).all()) and bool((out[5] == 0).all())


@pytest.mark.parametrize("dim,kv_heads,heads,seqs", [(64, 4, 8, 130), (128, 3, 6, 200), (256, 5, 5, 65), (128, 8, 8, 64)])
def test_decode_of_many_sequences_longest_first(dim, kv_heads, heads, seqs):
    """Whole rows by their lengths, in groups of 64: equal lengths, none, one far longer than the others."""
    lens = [(37 * b * b) % 211 if b % 5 else 96 for b in range(seqs)]
    lens[seqs // 2], lens[-1], lens[0] = 1900, 0, 1
    check_decode(Problem8(seqs, lens, heads, kv_heads, dim, 32, torch.float16), bound_len=2100)


def test_two_streams_at_once_with_workspaces_of_their_own():
    P, Q = Problem8(71, [9000], 8, 2, 128, 64, torch.bfloat16), Problem8(72, [700, 5000], 8, 2, 128, 64, torch.bfloat16)
    attn = tman.Attn(8, 0.09)
    calls = []
    for X in (P, Q):
        B, n = len(X.lens_list), max(X.lens_list)
        q = X.normal(B, 8, 128)
        want, got = torch.empty_like(q), torch.empty_like(q)
        spaces = [torch.zeros(tman.tman_attn_decode_kv8_workspace_bytes(X.cache, attn, n), dtype=torch.uint8, device=dev()) for _ in range(2)]
        tman.tman_attn_decode_kv8(X.cache, attn, q, X.lens, want, n, spaces[0])
        calls.append((tman.bound_attn_decode_kv8(X.cache, attn, q, X.lens, got, n, spaces[1]), torch.cuda.Stream(), want, got))
    torch.cuda.synchronize()
    for _ in range(30):
        for call, stream, _, _ in calls:
            call(stream.cuda_stream)
    torch.cuda.synchronize()
    for _, _, want, got in calls:
        assert torch.equal(want, got)  # the same bits every time


@pytest.mark.parametrize("dim,kv_heads,heads", [(128, 1, 1), (64, 2, 8), (256, 1, 4)])
def test_decode_long_lengths_in_many_pieces(dim, kv_heads, heads):
    P = Problem8(21, [20000, 1, 8191], heads, kv_heads, dim, 64, torch.bfloat16)
    _, ws = check_decode(P)
    check_decode(P, window=9000, cap=50.0, workspace=ws)
    check_decode(P, window=9000, bound_len=20001, workspace=None)


def test_seen_nan_is_seen_and_large_exponents_overflow_only_fp16():
    P = Problem8(2, [40, 40], 2, 1, 64, 16, torch.float16)
    page, slot = P.row(0, 20)
    P.v[page, 0, slot, 3] = 0x7f
    page, slot = P.row(1, 33)
    P.ve[page, 0, 0] = 140  # 448 * 2^13 is an infinity
    q = P.normal(2, 2, 64)
    out = torch.empty_like(q)
    attn = tman.Attn(2, 0.125)
    ws = torch.zeros(tman.tman_attn_decode_kv8_workspace_bytes(P.cache, attn, 40), dtype=torch.uint8, device=dev())
    tman.tman_attn_decode_kv8(P.cache, attn, q, P.lens, out, 40, ws)
    assert bool(torch.isnan(out[0, :, 3]).all()) and bool(torch.isfinite(out[0, :, 4:]).all())
    assert not bool(torch.isfinite(out[1]).all())
    B16 = tman.KvCache8(P.k, P.v, P.ke, P.ve, P.table, torch.bfloat16)
    out2 = torch.empty(2, 2, 64, dtype=torch.bfloat16, device=dev())
    tman.tman_attn_decode_kv8(B16, attn, q.bfloat16(), P.lens, out2, 40, ws)
    assert bool(torch.isfinite(out2[1]).all())


MASKS = ["causal", "documents", "prefix", "empty"]


def mask_of(kind, lens, new):
    first, end = [], []
    for n, t in zip(lens, new):
        for i in range(n - t, n):
            first.append({"documents": i // 37 * 37, "empty": n if i % 3 else 0}.get(kind, 0))
            end.append(max(i + 1, n * 3 // 4) if kind == "prefix" else i + 1)
    return (None if kind in ("causal", "prefix") else first), (end if kind == "prefix" else None)


# few rows (codes are read by the attention itself) and many (over a copy)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("heads,kv_heads,page", [(4, 4, 16), (6, 2, 64), (8, 1, 512)])
def test_few_rows(dtype, dim, mask, heads, kv_heads, page):
    lens, new = [5, 40, 0, 700, 129, 64, 3], [5, 3, 0, 9, 1, 17, 0]
    first, end = mask_of(mask, lens, new)
    P = Problem8(dim + heads, lens, heads, kv_heads, dim, page, dtype)
    check_prefill(P, new, first, end)


@pytest.mark.parametrize("dtype,dim,heads,kv_heads,page", [(torch.float16, 64, 8, 1, 16), (torch.bfloat16, 128, 4, 1, 64), (torch.float16, 256, 4, 2, 32),
                                                           (torch.bfloat16, 64, 2, 2, 1024)])
@pytest.mark.parametrize("mask", MASKS)
def test_many_rows(dtype, dim, heads, kv_heads, page, mask):
    lens, new = [2100, 0, 333, 2400], [1100, 0, 333, 700]
    first, end = mask_of(mask, lens, new)
    P = Problem8(dim, lens, heads, kv_heads, dim, page, dtype)
    check_prefill(P, new, first, end, sample=range(0, 1100, 97))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("many", [False, True])
def test_prompts_of_more_than_64_sequences(dim, many):
    lens = [(29 * b * b) % 150 + (b % 3 > 0) for b in range(140)]
    if many:
        lens[70] = 2600
    new = [0 if b % 7 == 3 else min(n, 1 + (13 * b) % (400 if many else 9)) for b, n in enumerate(lens)]
    if many:
        new = [min(n, 600) if b == 70 else n for b, n in enumerate(lens)]
        heads, kv_heads = 24, 1
    else:
        heads, kv_heads = 4, 2
    check_prefill(Problem8(dim, lens, heads, kv_heads, dim, 16, torch.float16), new, sample=[0, 99])


@pytest.mark.parametrize("rule", [dict(cap=20.0), dict(sloped=True), dict(window=1), dict(window=100, sloped=True), dict(window=5000), dict(scale=-0.3),
                                  dict(cap=1000.0)])
@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("dtype,dim,page", [(torch.float16, 128, 16), (torch.bfloat16, 64, 32), (torch.bfloat16, 256, 64)])
def test_prompt_rules(rule, many, dtype, dim, page):
    lens, new = ([2500, 70], [900, 70]) if many else ([600, 33, 1], [6, 33, 1])
    check_prefill(Problem8(31, lens, 4, 1, dim, page, dtype), new, sample=range(0, 900, 83), **rule)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_a_distance_bias_with_positions_ahead_of_the_queries(dim, cap):
    """A prefix seen by all, also ahead of a token: whole tiles on both sides of the queries, NaN where nobody looks."""
    lens, new = [1500, 900, 300], [1200, 900, 130]
    end = [max(i + 1, n * 5 // 6) for n, t in zip(lens, new) for i in range(n - t, n)]
    P = Problem8(dim + 1, lens, 4, 1, dim, 32, torch.bfloat16)
    check_prefill(P, new, end=end, cap=cap, sloped=True, sample=range(0, 1200, 71))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("many", [False, True])
def test_values_that_some_rows_must_not_see(dim, many):
    """NaN codes and blocks of overflowing exponents in places that only some rows see."""
    lens, new = ([2500], [900]) if many else ([300], [20])
    P = Problem8(41, lens, 4, 1, dim, 16, torch.float16)
    n, t = lens[0], new[0]
    bad = n - t // 2
    page, slot = P.row(0, bad)
    P.v[page, :, slot, 5], P.v[page, :, slot, dim - 1] = 0x7f, 0xff
    H = 4
    q = P.normal(t, H, dim)
    out = torch.empty_like(q)
    attn = tman.Attn(H, dim ** -0.5)
    need = tman.tman_attn_prefill_kv8_workspace_bytes(P.cache, attn, t, n)
    ws = torch.zeros(max(need, 16), dtype=torch.uint8, device=dev())
    tman.tman_attn_prefill_kv8(P.cache, attn, q, P.ints([0, t]), P.lens, out, n, ws)
    sees = torch.arange(n - t, n, device=dev()) >= bad
    assert bool(torch.isfinite(out[~sees]).all())
    nan = torch.isnan(out[sees])
    assert bool(nan[..., 5].all()) and bool(nan[..., dim - 1].all()) and not bool(nan[..., :5].any())


def test_one_workspace_for_calls_of_all_kinds():
    """Its tickets are at zero whatever ran before: the copy of a prompt, pieces of single tokens, few rows, both caches' functions."""
    P = Problem8(51, [6000, 900], 4, 1, 128, 64, torch.float16)
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device=dev())
    values = [ref.decode(x, e).half() for x, e in ((P.k, P.ke), (P.v, P.ve))]
    plain = tman.KvCache(*values, P.table)
    attn = tman.Attn(4, 0.1)
    for _ in range(2):
        check_decode(P, workspace=ws)
        check_prefill(P, [700, 900], workspace=ws, sample=range(0, 900, 211))
        q, out = P.normal(2, 4, 128), torch.empty(2, 4, 128, dtype=torch.float16, device=dev())
        tman.tman_attn_decode(plain, attn, q, P.lens, out, 6000, ws)
        again = torch.empty_like(out)
        tman.tman_attn_decode_kv8(P.cache, attn, q, P.lens, again, 6000, ws)
        assert bool(((out.double() - again.double()).abs() <= 2.0 ** -9 * (1 + out.abs().double())).all())
        check_prefill(P, [3, 9], workspace=ws)


def test_pages_and_lengths_out_of_range_stay_inside_and_are_reported():
    P = Problem8(61, [100, 64], 4, 2, 64, 16, torch.float16)
    attn = tman.Attn(4, 0.1)
    ws = torch.zeros(8 << 20, dtype=torch.uint8, device=dev())
    q = P.normal(2, 4, 64)
    out = torch.empty_like(q)
    P.table[0, 2] = 2 ** 30
    P.table[1, 0] = -7
    tman.tman_attn_decode_kv8(P.cache, attn, q, P.lens, out, 100, ws)
    assert tman.tman_device_status() == ERR_INDEX
    qs, outs = P.normal(20, 4, 64), torch.empty(20, 4, 64, dtype=torch.float16, device=dev())
    tman.tman_attn_prefill_kv8(P.cache, attn, qs, P.ints([0, 10, 20]), P.lens, outs, 100, ws)
    assert tman.tman_device_status() == ERR_INDEX
    tman.tman_attn_decode_kv8(P.cache, attn, q, P.ints([2 ** 31 - 1, -1]), out, 100, ws)
    assert tman.tman_device_status() == ERR_INDEX
    big = Problem8(62, [2500], 4, 1, 64, 16, torch.float16)
    big.table[0, 50] = 2 ** 30
    qb = big.normal(900, 4, 64)
    ob = torch.empty_like(qb)
    tman.tman_attn_prefill_kv8(big.cache, attn, qb, big.ints([0, 900]), big.lens, ob, 2500, ws)
    assert tman.tman_device_status() == ERR_INDEX and tman.tman_device_status() == 0


def test_a_side_stream_and_a_pool_beyond_4_gib():
    page, dim, G = 1024, 256, 8
    n_pages = 2100  # 4.4 GB of keys
    k = torch.zeros(n_pages, G, page, dim, dtype=torch.uint8, device=dev())
    v = torch.zeros_like(k)
    ke = torch.full((n_pages, G, page // 16), 120, dtype=torch.uint8, device=dev())
    ve = ke.clone()
    gen = torch.Generator(device=dev())
    gen.manual_seed(1)
    for p in (2099, 2098, 3):
        k[p], v[p] = ((torch.randn(G, page, dim, generator=gen, device=dev()) * 90).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
                      for _ in range(2))
    table = torch.tensor([[2099, 3, 2098]], dtype=torch.int32, device=dev())
    cache = tman.KvCache8(k, v, ke, ve, table, torch.bfloat16)
    n = 2500
    lens = torch.tensor([n], dtype=torch.int32, device=dev())
    q = torch.randn(1, G, dim, generator=gen, device=dev()).bfloat16()
    out = torch.empty_like(q)
    attn = tman.Attn(G, 0.05)
    ws = torch.zeros(tman.tman_attn_decode_kv8_workspace_bytes(cache, attn, n), dtype=torch.uint8, device=dev())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    tman.tman_attn_decode_kv8(cache, attn, q, lens, out, n, ws, stream=side)
    side.synchronize()
    rows = [ref.decode(x[table[0].long()], e[table[0].long()]).transpose(0, 1).reshape(G, -1, dim)[:, :n] for x, e in ((k, ke), (v, ve))]
    o, _, _, bound, _, _ = attend(q[0], *rows, n - 1, 0, n, 0.05, 0.0, None, 0, torch.bfloat16)
    within(out[0], o, bound, "out")
