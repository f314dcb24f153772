"""The key-value cache's operators against plain 64-bit forms: types, head sizes and groups, pages, lengths from none to several
pieces, masks that hide rows of tiles and whole rows, values that must not be seen, strides, streams, workspaces."""
import math

import pytest
import torch

import paper_2511_11248_amd as tman
from attention_ref import UNIT, attend, gather
from gpu_helpers import dev

pytestmark = pytest.mark.gpu
ERR_INDEX = -10
NAN, INF = float("nan"), float("inf")


class Problem:
    """Sequences of given lengths in a cache of shuffled pages; what lies behind a sequence's end, and pages of nobody, are NaN."""

    def __init__(self, seed, lens, heads, kv_heads, dim, page, dtype, extra=2, spare_pages=0, poison=NAN):
        self.gen = torch.Generator(device=dev())
        self.gen.manual_seed(seed)
        self.lens_list, self.heads, self.kv_heads, self.dim, self.page, self.dtype = lens, heads, kv_heads, dim, page, dtype
        wide = max(1, max((n + page - 1) // page for n in lens)) + 1
        n_pages = sum((n + page - 1) // page for n in lens) + extra + spare_pages
        order = torch.randperm(n_pages, generator=self.gen, device=dev()).tolist()
        self.k = self.normal(n_pages, kv_heads, page, dim)
        self.v = self.normal(n_pages, kv_heads, page, dim)
        own = torch.zeros(n_pages, page, dtype=torch.bool, device=dev())
        table = torch.full((len(lens), wide), 2 ** 30, dtype=torch.int32)  # unused entries are never used
        for b, n in enumerate(lens):
            for i in range((n + page - 1) // page):
                table[b, i] = order.pop()
                own[table[b, i], :n - i * page] = True
        self.spare = order
        hidden = ~own[:, None, :, None].expand_as(self.k)
        self.k[hidden], self.v[hidden] = poison, poison
        self.table, self.lens = table.to(dev()), self.ints(lens)
        self.cache = tman.KvCache(self.k, self.v, self.table)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.gen, device=dev()).to(self.dtype)

    def ints(self, x):
        return torch.tensor(x, dtype=torch.int32, device=dev())

    def slopes(self):
        return torch.tensor([2.0 ** (-8.0 * (h + 1) / self.heads) for h in range(self.heads)], dtype=torch.float32, device=dev())

    def row(self, b, j):
        """(page, slot) of position j of sequence b"""
        return int(self.table[b, j // self.page]), j % self.page


def within(got, want, bound, what):
    off = (got.double() - want).abs()
    ok = (off <= bound) | ((got.double() == want))
    assert bool(ok.all()), f"{what}: off by {(off / bound.clamp(min=1e-300))[~ok].max().item():.3g} of the bound"


def check_decode(P, first=None, cap=0.0, window=0, sloped=False, weights=False, scale=None, workspace=None, fused=True, bound_len=None):
    B, H, G, D = len(P.lens_list), P.heads, P.kv_heads, P.dim
    scale = D ** -0.5 if scale is None else scale
    qkv = P.normal(B, H + 2 * G, D)
    q = qkv[:, :H] if fused else qkv[:, :H].contiguous()
    out = torch.full((B, H + 1, D), 7.0, dtype=P.dtype, device=dev())[:, :H]
    lse = torch.full((B, H), NAN, device=dev())
    slopes = P.slopes() if sloped else None
    attn = tman.Attn(H, scale, cap=cap, window=window, slopes=slopes)
    max_len = bound_len or max(1, max(P.lens_list))
    w = w0 = None
    if weights:
        w = torch.rand(P.k.shape[:3], generator=P.gen, device=dev())
        w0 = w.clone()
    ws = workspace
    if ws is None:
        ws = torch.zeros(tman.tman_attn_decode_workspace_bytes(P.cache, attn, max_len, weights), dtype=torch.uint8, device=dev())
    firsts = None if first is None else P.ints(first)
    tman.tman_attn_decode(P.cache, attn, q, P.lens, out, max_len, ws, first=firsts, lse=lse, weights=w)
    assert tman.tman_device_status() == 0
    want_w = None if w is None else w0.double()
    for b, n in enumerate(P.lens_list):
        lo = 0 if first is None else max(first[b], 0)
        k, v = gather(P.k, P.table, b, n), gather(P.v, P.table, b, n)
        o, l, p, bound, l_bound, E = attend(q[b], k, v, n - 1, lo, n, scale, cap, slopes, window, P.dtype)
        within(out[b], o, bound, f"out[{b}], length {n}")
        within(lse[b], l, l_bound, f"lse[{b}], length {n}")
        if weights and n:
            add = p.view(G, H // G, n).sum(1)
            for i in range((n + P.page - 1) // P.page):
                part = add[:, i * P.page:(i + 1) * P.page]
                want_w[P.table[b, i].long(), :, :part.shape[1]] += part
    if weights:
        # every probability is off by 4 E of itself and fp32's roundings; sums of the group and with what was there
        tol = 2 * ((want_w - w0.double()).abs() * (4 * 2.0 ** -14 + 2.0 ** -18) + want_w.abs() * 2.0 ** -22)
        within(w, want_w, tol, "weights")
        same = want_w == w0.double()
        assert torch.equal(w[same], w0[same])
    return out, ws


LENS = [1, 0, 15, 16, 17, 31, 32, 33, 127, 128, 129, 300, 1027]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads,page", [(4, 4, 16), (6, 2, 32), (8, 1, 64), (20, 1, 128), (32, 2, 256), (5, 5, 1024)])
def test_decode_lengths(dtype, dim, heads, kv_heads, page):
    P = Problem(dim + heads, LENS, heads, kv_heads, dim, page, dtype)
    check_decode(P)


@pytest.mark.parametrize("dtype,dim,page", [(torch.float16, 64, 16), (torch.bfloat16, 128, 32), (torch.float16, 256, 64)])
@pytest.mark.parametrize("rule", [dict(cap=20.0), dict(sloped=True), dict(cap=30.0, sloped=True, weights=True), dict(weights=True),
                                  dict(window=1), dict(window=40), dict(window=333, cap=5.0, weights=True), dict(window=5000),
                                  dict(scale=-0.3), dict(scale=0.0)])
def test_decode_rules(dtype, dim, page, rule):
    P = Problem(3 + dim, [1, 0, 40, 41, 72, 500, 2049], 10, 2, dim, page, dtype)
    check_decode(P, **rule)


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
def test_decode_first_hides_leading_positions_whatever_they_hold(dim, weights):
    lens = [50, 50, 50, 50, 700, 700, 0, 3]
    first = [0, 7, 49, 50, 133, 900, 5, -4]  # also nothing left, beyond the end, before the start
    P = Problem(11, lens, 8, 2, dim, 16, torch.float16)
    for b, (n, f) in enumerate(zip(lens, first)):
        for j in range(0, min(max(f, 0), n)):
            page, slot = P.row(b, j)
            P.k[page, :, slot], P.v[page, :, slot] = (INF, NAN) if j % 2 else (NAN, -INF)
    out, _ = check_decode(P, first=first, weights=weights)
    assert bool((out[3] == 0).all()) and bool((out[5] == 0).all())


@pytest.mark.parametrize("dim,kv_heads,heads", [(128, 1, 1), (64, 2, 8), (256, 1, 4)])
def test_decode_long_lengths_in_many_pieces(dim, kv_heads, heads):
    P = Problem(21, [20000, 1, 8191], heads, kv_heads, dim, 64, torch.bfloat16)
    check_decode(P, weights=True)
    check_decode(P, window=9000, cap=50.0)


def test_decode_workspace_goes_from_call_to_call_of_any_sizes():
    ws = torch.zeros(16 << 20, dtype=torch.uint8, device=dev())
    for seed, (lens, heads, kv, dim) in enumerate([([3000], 8, 1, 128), ([100, 5000, 7], 4, 2, 64), ([900] * 9, 6, 6, 64), ([4000], 8, 1, 128)]):
        P = Problem(seed, lens, heads, kv, dim, 32, torch.float16)
        check_decode(P, weights=seed % 2 == 1, workspace=ws)
        check_decode(P, workspace=ws, bound_len=max(lens) + 1000 * seed)
    assert not ws[:4096 * 4].any()


def test_decode_visible_infinities_and_nan_stay_in_their_sequence_and_head():
    P = Problem(31, [200, 200, 200], 4, 2, 128, 16, torch.float16)
    page, slot = P.row(1, 77)
    P.v[page, 0, slot, 5] = INF
    P.k[page, 1, slot] = NAN
    B, H, D = 3, 4, 128
    q, out, clean = P.normal(B, H, D), torch.empty(B, H, D, dtype=P.dtype, device=dev()), torch.empty(B, H, D, dtype=P.dtype, device=dev())
    attn = tman.Attn(H, D ** -0.5)
    ws = torch.zeros(tman.tman_attn_decode_workspace_bytes(P.cache, attn, 200), dtype=torch.uint8, device=dev())
    tman.tman_attn_decode(P.cache, attn, q, P.lens, out, 200, ws)
    P.v[page, 0, slot, 5], P.k[page, 1, slot] = 0.0, 0.0
    tman.tman_attn_decode(P.cache, attn, q, P.lens, clean, 200, ws)
    assert torch.equal(out[0], clean[0]) and torch.equal(out[2], clean[2])
    assert bool((out[1, :2, 5] == INF).all()) and bool(out[1, 2:].isnan().all())
    keep = [d for d in range(D) if d != 5]
    assert bool(out[1, :2][:, keep].isfinite().all())


def test_results_are_the_same_every_time_and_on_another_stream():
    P = Problem(41, [5000, 17, 1234], 8, 2, 128, 32, torch.float16)
    attn = tman.Attn(8, 0.09, cap=30.0)
    q, out, again = P.normal(3, 8, 128), *(torch.empty(3, 8, 128, dtype=P.dtype, device=dev()) for _ in range(2))
    need = tman.tman_attn_decode_workspace_bytes(P.cache, attn, 5000, True)
    ws = torch.zeros(need, dtype=torch.uint8, device=dev())
    w, w2 = (torch.zeros(P.k.shape[:3], device=dev()) for _ in range(2))
    tman.tman_attn_decode(P.cache, attn, q, P.lens, out, 5000, ws, weights=w)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for k in range(4):
        w2.zero_()
        again.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            tman.tman_attn_decode(P.cache, attn, q, P.lens, again, 5000, ws, weights=w2, stream=s if k % 2 else None)
        s.synchronize()
        assert torch.equal(out, again) and torch.equal(w, w2)


def test_decode_in_a_graph():
    P = Problem(43, [3000, 64], 8, 2, 64, 16, torch.float16)
    attn = tman.Attn(8, 0.125)
    q, out, want = P.normal(2, 8, 64), *(torch.empty(2, 8, 64, dtype=P.dtype, device=dev()) for _ in range(2))
    ws = torch.zeros(tman.tman_attn_decode_workspace_bytes(P.cache, attn, 4000), dtype=torch.uint8, device=dev())
    tman.tman_attn_decode(P.cache, attn, q, P.lens, out, 4000, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tman.tman_attn_decode(P.cache, attn, q, P.lens, out, 4000, ws)
    for n in ([3000, 64], [2999, 1], [31, 0], [3000, 33]):  # lengths are read when the graph runs
        P.lens.copy_(P.ints(n))
        q.copy_(P.normal(2, 8, 64))
        tman.tman_attn_decode(P.cache, attn, q, P.lens, want, 4000, ws)
        torch.cuda.synchronize()
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


# ---- prompts

def check_prefill(P, new, first=None, end=None, cap=0.0, window=0, sloped=False, scale=None, rows=None, workspace=None, bound_len=None):
    """`new` tokens of every sequence are the last of it; rows: how many randomly chosen tokens are compared (None: all)."""
    H, G, D, N = P.heads, P.kv_heads, P.dim, sum(new)
    scale = D ** -0.5 if scale is None else scale
    q = P.normal(N, H + 2 * G, D)[:, :H]
    out = torch.full((N, H + 1, D), 7.0, dtype=P.dtype, device=dev())[:, 1:]
    lse = torch.full((N, H), NAN, device=dev())
    starts = [0]
    for t in new:
        starts.append(starts[-1] + t)
    slopes = P.slopes() if sloped else None
    attn = tman.Attn(H, scale, cap=cap, window=window, slopes=slopes)
    max_len = bound_len or max(P.lens_list)
    need = tman.tman_attn_prefill_workspace_bytes(P.cache, attn, N, max_len)
    ws = workspace if workspace is not None else torch.zeros(need, dtype=torch.uint8, device=dev()) if need else None
    tman.tman_attn_prefill(P.cache, attn, q, P.ints(starts), P.lens, out, max_len, ws, first=None if first is None else P.ints(first),
                           end=None if end is None else P.ints(end), lse=lse)
    assert tman.tman_device_status() == 0
    r = torch.Generator()
    r.manual_seed(N)
    for b, (t, n) in enumerate(zip(new, P.lens_list)):
        k, v = gather(P.k, P.table, b, n), gather(P.v, P.table, b, n)
        chosen = range(t) if rows is None or t <= rows else sorted({0, t - 1, *torch.randint(t, (rows,), generator=r).tolist()})
        for i in chosen:
            x, at = starts[b] + i, n - t + i
            lo = 0 if first is None else max(first[x], 0)
            hi = min(at + 1 if end is None else end[x], n)
            o, l, _, bound, l_bound, _ = attend(q[x], k, v, at, lo, hi, scale, cap, slopes, window, P.dtype)
            within(out[x], o, bound, f"out, sequence {b}, token {i} of {t}, [{lo}, {hi})")
            within(lse[x], l, l_bound, f"lse, sequence {b}, token {i} of {t}")
    return out, lse


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads,page", [(2, 2, 16), (6, 2, 32), (7, 1, 64), (20, 1, 256)])
def test_prefill_lengths(dtype, dim, heads, kv_heads, page):
    new = [1, 0, 2, 31, 33, 5, 65, 1, 7]
    past = [0, 9, 0, 0, 0, 60, 63, 300, 129]
    P = Problem(dim + heads, [t + p for t, p in zip(new, past)], heads, kv_heads, dim, page, dtype)
    check_prefill(P, new)


@pytest.mark.parametrize("dtype,dim,page", [(torch.float16, 64, 16), (torch.bfloat16, 128, 32), (torch.float16, 256, 64)])
@pytest.mark.parametrize("rule", [dict(cap=20.0), dict(sloped=True), dict(cap=30.0, sloped=True), dict(window=1), dict(window=50),
                                  dict(window=64, cap=3.0), dict(scale=-0.4), dict(scale=0.0)])
def test_prefill_rules(dtype, dim, page, rule):
    P = Problem(5 + dim, [150, 90, 260], 6, 2, dim, page, dtype)
    check_prefill(P, [150, 1, 77], rows=40, **rule)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("sloped,window", [(False, 0), (True, 0), (False, 30)])
def test_prefill_intervals(dim, sloped, window):
    new, lens = [200, 70], [200, 400]
    P = Problem(9, lens, 4, 2, dim, 16, torch.float16)
    first, end = [], []
    for t, n in zip(new, lens):
        for i in range(n - t, n):
            kind = i % 5
            first.append([0, i // 3, i, n, -5][kind])             # from the start, inside, itself alone, nothing, before the start
            end.append([i + 1, n - 1, i + 1, n + 9, n + 100][kind])  # causal, ahead of the query, ..., beyond the end
    check_prefill(P, new, first=first, end=end, sloped=sloped, window=window)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_prefill_documents_hide_each_other_whatever_they_hold(dtype, dim):
    """Documents behind one another, one of them full of infinities and NaN: the others do not notice; padding sees nothing."""
    n, starts = 300, [0, 70, 101, 102, 230]
    P = Problem(13, [n], 4, 2, dim, 32, dtype)
    first = [max(s for s in starts if s <= i) for i in range(n)]
    first[-6:] = [n] * 6
    q_state = P.gen.get_state()
    want, want_lse = check_prefill(P, [n], first=first)
    for j in range(102, 230):
        page, slot = P.row(0, j)
        P.k[page, :, slot] = [NAN, INF, -INF][j % 3]
        P.v[page, :, slot] = [-INF, NAN, INF][j % 3]
    H, D = 4, dim
    P.gen.set_state(q_state)
    q = P.normal(n, H + 4, D)[:, :H]
    out, lse = torch.empty(n, H, D, dtype=dtype, device=dev()), torch.empty(n, H, device=dev())
    attn = tman.Attn(H, D ** -0.5)
    ws = torch.zeros(tman.tman_attn_prefill_workspace_bytes(P.cache, attn, n, n), dtype=torch.uint8, device=dev())
    tman.tman_attn_prefill(P.cache, attn, q, P.ints([0, n]), P.lens, out, n, ws, first=P.ints(first), lse=lse)
    good = [i for i in range(n) if not 102 <= i < 230]
    assert torch.equal(out[good], want[good]) and torch.equal(lse[good], want_lse[good])
    assert bool((out[-6:] == 0).all()) and bool((lse[-6:] == -INF).all())


def test_prefill_one_infinite_value_reaches_those_that_see_it_and_nobody_else():
    n, H, D = 100, 2, 64
    P = Problem(15, [n], H, 1, D, 16, torch.float16)
    q, out, clean = P.normal(n, H, D), *(torch.empty(n, H, D, dtype=torch.float16, device=dev()) for _ in range(2))
    attn = tman.Attn(H, D ** -0.5)
    ws = torch.zeros(max(1, tman.tman_attn_prefill_workspace_bytes(P.cache, attn, n, n)), dtype=torch.uint8, device=dev())
    run = lambda to: tman.tman_attn_prefill(P.cache, attn, q, P.ints([0, n]), P.lens, to, n, ws)  # noqa: E731
    run(clean)
    page, slot = P.row(0, 40)
    P.v[page, 0, slot, 9] = -INF
    run(out)
    assert torch.equal(out[:40], clean[:40])
    assert bool((out[40:, :, 9] == -INF).all())
    keep = [d for d in range(D) if d != 9]
    assert bool(out[40:][:, :, keep].isfinite().all())
    within(out[40:][:, :, keep], clean[40:][:, :, keep].double(), 2 * UNIT[torch.float16] * clean[40:][:, :, keep].double().abs() + 1e-6, "rest")


@pytest.mark.parametrize("dtype,dim,heads,kv_heads", [(torch.float16, 128, 8, 2), (torch.bfloat16, 64, 3, 3), (torch.float16, 256, 4, 1)])
def test_prefill_long(dtype, dim, heads, kv_heads):
    P = Problem(17, [1500, 3000], heads, kv_heads, dim, 64, dtype)
    check_prefill(P, [1500, 700], rows=25, cap=25.0)
    check_prefill(P, [1500, 700], rows=25, sloped=True, end=[1000 if i < 1000 else i + 1 for i in range(1500)] + [1 << 30] * 700)


@pytest.mark.parametrize("tokens", [1, 3, 40])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_prefill_few_tokens_of_a_long_cache_in_many_pieces(tokens, dim):
    P = Problem(19, [9000, 64, 5000], 4, 1, dim, 16, torch.float16)
    check_prefill(P, [tokens, 1, tokens], rows=10)
    check_prefill(P, [tokens, 0, tokens], rows=10, window=3000, first=[4000] * tokens + [5000] * tokens)


def test_prefill_workspace_goes_from_call_to_call_of_any_sizes():
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device=dev())
    for seed, (lens, new) in enumerate([([4000], [9]), ([100, 5000, 7], [100, 1, 0]), ([300] * 9, [30] * 9), ([4000], [5])]):
        P = Problem(seed, lens, 4, 2, 64, 32, torch.float16)
        check_prefill(P, new, rows=5, workspace=ws)
        check_decode(P, workspace=ws)
    assert not ws[:4096 * 4].any()


def test_many_sequences():
    """More sequences than lanes of a wave, some without new tokens."""
    new = [(b * 7) % 5 for b in range(150)]
    P = Problem(23, [t + b % 40 for b, t in enumerate(new)], 4, 2, 64, 16, torch.float16)
    check_prefill(P, new)
    check_decode(P)


def test_prefill_agrees_with_decode_token_by_token():
    """A prompt of one token is what decode does (the two add up in different orders)."""
    P = Problem(25, [1000, 37], 8, 2, 128, 16, torch.float16)
    q, a, b = P.normal(2, 8, 128), *(torch.empty(2, 8, 128, dtype=torch.float16, device=dev()) for _ in range(2))
    attn = tman.Attn(8, 0.1, cap=10.0, window=700)
    ws = torch.zeros(32 << 20, dtype=torch.uint8, device=dev())
    tman.tman_attn_decode(P.cache, attn, q, P.lens, a, 1000, ws)
    tman.tman_attn_prefill(P.cache, attn, q, P.ints([0, 1, 2]), P.lens, b, 1000, ws)
    # each within its own bound of the same exact result
    for s, n in enumerate([1000, 37]):
        *_, bound, _, _ = attend(q[s], gather(P.k, P.table, s, n), gather(P.v, P.table, s, n), n - 1, 0, n, 0.1, 10.0, None, 700, P.dtype)
        within(a[s], b[s].double(), 2 * bound, "decode against prefill")


# ---- offsets beyond 32 bits, indices out of range

def test_a_pool_of_more_than_4_gib():
    page, G, D = 256, 2, 256
    n_pages = (4 << 30) // (page * G * D * 2) + 40
    k = torch.empty(n_pages, G, page, D, dtype=torch.float16, device=dev())
    v = torch.empty_like(k)
    P = Problem(27, [600, 300], 4, G, D, page, torch.float16)
    used = [x for b, n in enumerate([600, 300]) for x in P.table[b, :(n + page - 1) // page].tolist()]
    place = {x: n_pages - 1 - 7 * i for i, x in enumerate(used)}
    for x, y in place.items():
        k[y], v[y] = P.k[x], P.v[x]
    for b, n in enumerate([600, 300]):
        for i in range((n + page - 1) // page):
            P.table[b, i] = place[int(P.table[b, i])]
    P.k, P.v, P.cache = k, v, tman.KvCache(k, v, P.table)
    check_decode(P)
    check_prefill(P, [20, 300], rows=20)
    kn = P.normal(2, G, D)
    tman.tman_rope_append(P.cache, None, kn, -kn, P.lens, None)
    for b, n in enumerate([600, 300]):
        y, slot = P.row(b, n - 1)
        assert torch.equal(k[y, :, slot], kn[b]) and torch.equal(v[y, :, slot], -kn[b])


def test_indices_out_of_range_are_cut_and_reported():
    P = Problem(29, [100, 100], 4, 2, 64, 16, torch.float16, poison=0.0)
    H, D = 4, 64
    attn = tman.Attn(H, 0.1)
    ws = torch.zeros(32 << 20, dtype=torch.uint8, device=dev())
    q, out = P.normal(2, H, D), torch.empty(2, H, D, dtype=torch.float16, device=dev())
    starts, wide = P.ints([0, 1, 2]), P.table.shape[1] * 16
    decode = lambda n: tman.tman_attn_decode(P.cache, attn, q, P.lens, out, n, ws)  # noqa: E731
    prefill = lambda n: tman.tman_attn_prefill(P.cache, attn, q, starts, P.lens, out, n, ws)  # noqa: E731
    good = P.table.clone()
    for call in (decode, prefill):
        call(100)
        assert tman.tman_device_status() == 0
        call(99)  # a length beyond the caller's bound
        assert tman.tman_device_status() == ERR_INDEX and tman.tman_device_status() == 0
        P.lens.copy_(P.ints([100, wide + 1]))  # beyond the table; its last entries are of nobody
        call(1000)
        assert tman.tman_device_status() == ERR_INDEX
        P.lens.copy_(P.ints([-3, 100]))
        call(100)
        assert tman.tman_device_status() == ERR_INDEX and bool((out[0] == 0).all())
        P.lens.copy_(P.ints([100, 100]))
        for bad in (-1, P.k.shape[0], 2 ** 31 - 1):
            P.table[1, 2] = bad
            call(100)
            assert tman.tman_device_status() == ERR_INDEX
            P.table.copy_(good)
    kn = P.normal(2, 2, D)
    before = P.k.clone(), P.v.clone()
    for lens in ([0, 0], [wide + 1, -5]):
        P.lens.copy_(P.ints(lens))
        tman.tman_rope_append(P.cache, None, kn, kn, P.lens, None)
        assert tman.tman_device_status() == ERR_INDEX
        assert torch.equal(P.k, before[0]) and torch.equal(P.v, before[1])


# ---- rotary positions and append

def angles(n_pos, rot):
    pos = torch.arange(n_pos, dtype=torch.float64, device=dev())
    freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=dev()) / rot)
    a = pos[:, None] * freq
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def rotated(x, cs, rot, interleaved):
    """x [heads, dim], cs [rot / 2, 2], in 64 bits; and the sum of the magnitudes that meet in each element."""
    x, y = x.double(), x.double().clone()
    size = x.abs().clone()
    c, s = cs[:, 0].double(), cs[:, 1].double()
    i = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    j = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    y[:, i], y[:, j] = x[:, i] * c - x[:, j] * s, x[:, i] * s + x[:, j] * c
    size[:, i], size[:, j] = (x[:, i] * c).abs() + (x[:, j] * s).abs(), (x[:, i] * s).abs() + (x[:, j] * c).abs()
    return y, size


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,rot,sections,interleaved", [
    (64, 64, None, False), (64, 16, None, True), (128, 128, (16, 24, 24), False), (128, 64, (20, 12), True), (128, 48, (0, 24), False),
    (256, 256, (64, 0, 64), True), (256, 240, (1, 2, 117), False), (64, 0, None, False)])
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (9, 3), (0, 2), (40, 1)])
def test_append(dtype, dim, rot, sections, interleaved, heads, kv_heads):
    new, lens = [3, 0, 40, 1, 1], [3, 5, 100, 1, 33]
    P = Problem(33 + dim, lens, max(heads, 1), kv_heads, dim, 16, dtype)
    N, H, G = sum(new), heads, kv_heads
    qkv = P.normal(N, H + 2 * G, dim)
    q, k, v = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
    q_out = torch.full((N, H + 1, dim), 7.0, dtype=dtype, device=dev())
    starts = [sum(new[:b]) for b in range(len(new) + 1)]
    n_pos = 150
    rope = tman.Rope(angles(n_pos, rot), sections, interleaved) if rot else None
    axes = len(sections) if sections else 1
    positions = None
    if rope is not None and axes > 1:
        positions = torch.randint(n_pos, (axes, N), generator=P.gen, device=dev()).to(torch.int32)
    w = torch.rand(P.k.shape[:3], generator=P.gen, device=dev())
    k0, v0, w0 = P.k.clone(), P.v.clone(), w.clone()
    tman.tman_rope_append(P.cache, q if H else None, k, v, P.lens, q_out[:, :H] if H else None, rope=rope, positions=positions,
                          q_start=P.ints(starts), weights=w)
    assert tman.tman_device_status() == 0
    assert bool((q_out[:, H] == 7).all())
    axis = [a for a, count in enumerate(sections or (rot // 2,)) for _ in range(count)]
    written = torch.zeros(P.k.shape[0], P.page, dtype=torch.bool, device=dev())
    for b in range(len(new)):
        for i in range(new[b]):
            x, at = starts[b] + i, lens[b] - new[b] + i
            page, slot = P.row(b, at)
            written[page, slot] = True
            assert torch.equal(P.v[page, :, slot], v[x]) and bool((w[page, :, slot] == 0).all())
            if rope is None:
                assert torch.equal(P.k[page, :, slot], k[x]) and (not H or torch.equal(q_out[x, :H], q[x]))
                continue
            pos = [at] if positions is None else positions[:, x].tolist()
            cs = torch.stack([rope.cos_sin[pos[a], p] for p, a in enumerate(axis)])
            for got, of in ((P.k[page, :, slot], k[x]), (q_out[x, :H], q[x])):
                want, size = rotated(of, cs, rot, interleaved)
                # one rounding of the result, two or three of fp32 before it
                within(got, want, UNIT[dtype] * want.abs() + 2.0 ** -22 * size + 2.0 ** -25, "rotated")
                assert torch.equal(got[:, rot:], of[:, rot:])
    keep = ~written
    for got, was in ((P.k, k0), (P.v, v0)):
        assert torch.equal(got.transpose(1, 2)[keep].view(torch.int16), was.transpose(1, 2)[keep].view(torch.int16))
    assert torch.equal(w.transpose(1, 2)[keep], w0.transpose(1, 2)[keep])


def test_append_in_place_one_token_each_and_tokens_of_nobody():
    P = Problem(35, [1, 17, 64, 30], 6, 2, 128, 32, torch.float16)
    rope = tman.Rope(angles(64, 128))
    q, k = P.normal(4, 6, 128), P.normal(4, 2, 128)
    want = torch.empty_like(q)
    tman.tman_rope_append(P.cache, q, k, k, P.lens, want, rope=rope)
    tman.tman_rope_append(P.cache, q, k, k, P.lens, q, rope=rope)
    assert torch.equal(q, want)
    # q_start ends before the last token: it belongs to no sequence and nothing of it is written
    out = torch.full_like(q, 5.0)
    before = P.k.clone()
    tman.tman_rope_append(P.cache, q, k, k, P.ints([1, 17, 64, 29]), out, rope=rope, q_start=P.ints([0, 1, 2, 3, 3]))
    assert tman.tman_device_status() == 0
    assert bool((out[3] == 5).all()) and bool((out[:3] != 5).any())
    assert torch.equal(P.k.view(torch.int16), before.view(torch.int16))
    # a position that the table of angles has not
    tman.tman_rope_append(P.cache, q, k, k, P.lens, out, rope=tman.Rope(angles(63, 128)))
    assert tman.tman_device_status() == ERR_INDEX


# ---- eviction

def check_evict(P, weights, keep, recent, max_len=None):
    B, G, page = len(P.lens_list), P.kv_heads, P.page
    pages = (keep + page - 1) // page
    spare = list(P.spare)
    new_table = P.ints([[spare.pop() for _ in range(pages)] for _ in range(B)])
    kept = torch.full((B, G, keep), 99, dtype=torch.int32, device=dev())
    new_lens = torch.full((B,), 99, dtype=torch.int32, device=dev())
    k0, v0, w0 = P.k.clone(), P.v.clone(), weights.clone()
    tman.tman_kv_evict(P.cache, weights, P.lens, keep, recent, new_table, new_lens, kept, max_len or max(1, max(P.lens_list)))
    assert tman.tman_device_status() == 0
    assert new_lens.tolist() == [min(n, keep) for n in P.lens_list]
    untouched = torch.ones(P.k.shape[0], G, page, dtype=torch.bool, device=dev())
    for b, n in enumerate(P.lens_list):
        for g in range(G):
            at = [P.row(b, j) for j in range(n)]
            w = [float(w0[p, g, s]) for p, s in at]
            if n <= keep:
                want = list(range(n))
            else:
                order = sorted(range(n - recent), key=lambda j: (0 if w[j] != w[j] else 1, -w[j] if w[j] == w[j] else 0, j))
                want = sorted(order[:keep - recent]) + list(range(n - recent, n))
            assert kept[b, g].tolist() == want + [-1] * (keep - len(want))
            if want:
                src, slot = (torch.tensor([at[j][x] for j in want], device=dev()) for x in (0, 1))
                r = torch.arange(len(want), device=dev())
                dst = new_table[b].long()[r // page]
                bits = lambda t: t.view(torch.int16)  # noqa: E731
                assert torch.equal(bits(P.k[dst, g, r % page]), bits(k0[src, g, slot]))
                assert torch.equal(bits(P.v[dst, g, r % page]), bits(v0[src, g, slot]))
                assert torch.equal(weights[dst, g, r % page].view(torch.int32), w0[src, g, slot].view(torch.int32))
                untouched[dst, g, r % page] = False
    for got, was in ((P.k, k0), (P.v, v0)):
        assert torch.equal(got[untouched].view(torch.int16), was[untouched].view(torch.int16))
    assert torch.equal(weights[untouched].view(torch.int32), w0[untouched].view(torch.int32))


@pytest.mark.parametrize("dtype,dim", [(torch.float16, 64), (torch.bfloat16, 128), (torch.float16, 256)])
@pytest.mark.parametrize("keep,recent,page", [(1, 0, 16), (1, 1, 16), (64, 0, 16), (100, 30, 32), (100, 100, 64), (257, 1, 128), (900, 200, 16)])
def test_evict(dtype, dim, keep, recent, page):
    lens = [1000, 0, keep, keep + 1, 17, 333]
    P = Problem(keep + dim, lens, 2, 2, dim, page, dtype, spare_pages=len(lens) * ((keep + page - 1) // page))
    check_evict(P, torch.rand(P.k.shape[:3], generator=P.gen, device=dev()), keep, recent)


@pytest.mark.parametrize("kind", ["ties", "zeros", "negative", "special", "close"])
def test_evict_odd_weights(kind):
    lens, keep = [700, 200, 65], 64
    P = Problem(47, lens, 2, 2, 64, 16, torch.float16, spare_pages=12)
    w = torch.rand(P.k.shape[:3], generator=P.gen, device=dev())
    if kind == "ties":
        w = (w * 4).floor()
    elif kind == "zeros":
        w = torch.where(w < 0.5, 0.0, -0.0) * torch.ones_like(w)
    elif kind == "negative":
        w = w - 0.9
    elif kind == "close":
        w = 1.0 + (w * 8).floor() * 2.0 ** -23  # differ in the last bits alone
    else:
        w = torch.where(w < 0.03, torch.full_like(w, NAN), w)
        w = torch.where((w > 0.1) & (w < 0.13), torch.full_like(w, INF), w)
        w = torch.where((w > 0.2) & (w < 0.6), torch.full_like(w, -INF), w)
    check_evict(P, w, keep, 10)


def test_evict_long():
    P = Problem(49, [40000, 33000], 1, 1, 64, 128, torch.float16, spare_pages=2 * 79)
    check_evict(P, torch.rand(P.k.shape[:3], generator=P.gen, device=dev()), 10000, 33, max_len=50000)


def test_accumulate_evict_and_go_on():
    """What a program does: steps that add up weights, an eviction, steps on what was kept."""
    lens, keep, page, H, G, D = [300, 120], 100, 16, 4, 2, 64
    P = Problem(51, lens, H, G, D, page, torch.float16, spare_pages=2 * 8)
    w = torch.zeros(P.k.shape[:3], device=dev())
    attn = tman.Attn(H, D ** -0.5)
    ws = torch.zeros(tman.tman_attn_decode_workspace_bytes(P.cache, attn, 300, True), dtype=torch.uint8, device=dev())
    out = torch.empty(2, H, D, dtype=torch.float16, device=dev())
    total = 0
    for _ in range(3):
        tman.tman_attn_decode(P.cache, attn, P.normal(2, H, D), P.lens, out, 300, ws, weights=w)
        total += 1
    assert abs(float(w.double().sum()) - total * 2 * H) < 1e-3  # every row of probabilities adds up to one
    spare = list(P.spare)
    new_table = P.ints([[spare.pop() for _ in range(8)] for _ in range(2)])
    new_lens, kept = P.ints([0, 0]), torch.empty(2, G, keep, dtype=torch.int32, device=dev())
    tman.tman_kv_evict(P.cache, w, P.lens, keep, 20, new_table, new_lens, kept, 300)
    cache = tman.KvCache(P.k, P.v, new_table)
    lens2 = new_lens + 1
    q, kv = P.normal(2, H, D), P.normal(2, G, D)
    tman.tman_rope_append(cache, q, kv, kv, lens2, q, weights=w)
    tman.tman_attn_decode(cache, attn, q, lens2, out, keep + 1, ws, weights=w)
    assert tman.tman_device_status() == 0
    for b in range(2):
        k = torch.cat([gather(P.k, P.table, b, lens[b])[g][kept[b, g].long()][None] for g in range(G)])
        v = torch.cat([gather(P.v, P.table, b, lens[b])[g][kept[b, g].long()][None] for g in range(G)])
        k, v = torch.cat([k, kv[b][:, None].double()], 1), torch.cat([v, kv[b][:, None].double()], 1)
        o, _, _, bound, _, _ = attend(q[b], k, v, keep, 0, keep + 1, D ** -0.5, 0.0, None, 0, torch.float16)
        within(out[b], o, bound, "after the eviction")
