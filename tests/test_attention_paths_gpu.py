"""Prompt attention where one kernel hands over to another: up to and beyond 128 rows a sequence, short and long bounds, one piece and
several, a second kernel for the join or none; in graphs; the same bits every time.  The references and bounds are those of
test_attention_gpu.py."""
import pytest
import torch

import paper_2511_11248_amd as tman
from gpu_helpers import dev
from test_attention_gpu import Problem, check_decode, check_prefill

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("tokens,length,heads,kv_heads", [
    (8, 4096, 8, 1), (9, 4096, 8, 1),                # 64 and 72 rows: few, joined by the last workgroup or a second kernel
    (16, 4096, 8, 1), (17, 4096, 8, 1),              # 128 and 136 rows: few, many
    (2, 3000, 4, 1), (3, 3000, 4, 1),                # 8 and 12 rows a sequence
    (600, 2048, 4, 4), (600, 2049, 4, 4),            # the bound up to which short sequences go to the kernel for few rows
    (33, 33, 4, 4), (129, 129, 1, 1), (1, 1, 1, 1),
    (700, 6000, 2, 1), (257, 8192, 2, 2),            # many rows in pieces
])
def test_hand_overs(dim, tokens, length, heads, kv_heads):
    P = Problem(tokens + dim, [length], heads, kv_heads, dim, 32, torch.float16)
    check_prefill(P, [tokens], rows=8)
    check_prefill(P, [tokens], rows=8, cap=20.0, sloped=True, window=length // 2 + 1)


@pytest.mark.parametrize("page", [16, 1024])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_masks_at_every_edge_of_a_tile(dim, page):
    """Intervals that begin and end at, before and behind multiples of 32 and 64, for both kernels."""
    n = 320
    edges = [0, 1, 31, 32, 33, 63, 64, 65, 95, 96, 127, 128, 129, 191, 192, 255, 256, 319, 320]
    for tokens in (20, 150):
        P = Problem(dim + tokens, [n], 4, 1, dim, page, torch.bfloat16)
        pairs = [(a, b) for a in edges for b in edges if a <= b]
        first = [pairs[(7 * i) % len(pairs)][0] for i in range(tokens)]
        end = [pairs[(7 * i) % len(pairs)][1] for i in range(tokens)]
        check_prefill(P, [tokens], first=first, end=end)
        # the second kernel of many rows at the same masks
        long = Problem(dim + tokens, [n + 6000], 4, 1, dim, page, torch.bfloat16)
        check_prefill(long, [tokens], first=[a + 3000 for a in first], end=[b + 3000 for b in end], rows=30)


def test_every_row_hidden():
    for tokens, length in ((3, 50), (200, 3000)):
        P = Problem(3, [length], 4, 2, 128, 16, torch.float16)
        out, lse = check_prefill(P, [tokens], first=[length] * tokens, rows=4)
        assert bool((out == 0).all()) and bool((lse == -float("inf")).all())
    P = Problem(4, [5, 0, 700], 4, 2, 128, 16, torch.float16)
    out, _ = check_decode(P, first=[5, 0, 700])
    assert bool((out == 0).all())


@pytest.mark.parametrize("tokens,length,heads,kv_heads,dim", [(5, 5000, 8, 2, 64), (30, 3000, 8, 2, 128), (300, 9000, 4, 1, 128), (900, 900, 8, 8, 64),
                                                              (200, 5000, 2, 1, 256)])
def test_graphs_and_the_same_bits_every_time(tokens, length, heads, kv_heads, dim):
    P = Problem(51, [length], heads, kv_heads, dim, 64, torch.float16)
    attn = tman.Attn(heads, dim ** -0.5, cap=30.0, slopes=P.slopes())
    q, out, want = P.normal(tokens, heads, dim), *(torch.empty(tokens, heads, dim, dtype=P.dtype, device=dev()) for _ in range(2))
    need = tman.tman_attn_prefill_workspace_bytes(P.cache, attn, tokens, length)
    ws = torch.zeros(max(need, 16), dtype=torch.uint8, device=dev())
    starts = P.ints([0, tokens])
    run = lambda to: tman.tman_attn_prefill(P.cache, attn, q, starts, P.lens, to, length, ws)  # noqa: E731
    run(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(out)
    for n in (length, max(tokens, length - 1), tokens, length):  # lengths are read when the graph runs
        P.lens.copy_(P.ints([n]))
        q.copy_(P.normal(tokens, heads, dim))
        run(want)
        torch.cuda.synchronize()
        for _ in range(2):
            out.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
    assert tman.tman_device_status() == 0


def test_append_prompt_and_eviction_in_a_graph():
    """A chain of calls as one graph, replayed against the calls themselves."""
    H, G, D, page, keep = 4, 2, 64, 16, 64
    P = Problem(53, [200, 77], H, G, D, page, torch.float16, spare_pages=8, poison=0.0)
    w = torch.rand(P.k.shape[:3], generator=P.gen, device=dev())
    spare = list(P.spare)
    new_table = P.ints([[spare.pop() for _ in range(4)] for _ in range(2)])
    new_lens, kept = P.ints([0, 0]), torch.empty(2, G, keep, dtype=torch.int32, device=dev())
    attn = tman.Attn(H, 0.125)
    q, k, v = P.normal(5, H, D), P.normal(5, G, D), P.normal(5, G, D)
    out = torch.empty(5, H, D, dtype=torch.float16, device=dev())
    starts = P.ints([0, 3, 5])
    ws = torch.zeros(32 << 20, dtype=torch.uint8, device=dev())

    def chain():
        tman.tman_rope_append(P.cache, q, k, v, P.lens, out, q_start=starts, weights=w)
        tman.tman_attn_prefill(P.cache, attn, q, starts, P.lens, out, 200, ws)
        tman.tman_kv_evict(P.cache, w, P.lens, keep, 10, new_table, new_lens, kept, 200)

    def state():
        return [t.clone() for t in (out, P.k, P.v, w, new_lens, kept)]

    chain()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for _ in range(3):
        for t in (q, k, v):
            t.copy_(P.normal(*t.shape))
        w.copy_(torch.rand(w.shape, generator=P.gen, device=dev()))
        w0 = w.clone()
        chain()
        torch.cuda.synchronize()
        want = state()
        w.copy_(w0)
        out.zero_()
        kept.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(state(), want))
    assert tman.tman_device_status() == 0


def test_bound_calls_do_what_the_calls_do():
    """Checked once, run every step: the same bits as the calls, on the stream that they are given, refusals at once."""
    H, G, D, B = 6, 2, 128, 3
    P = Problem(55, [40, 700, 9], H, G, D, 32, torch.float16, poison=0.0)
    attn = tman.Attn(H, 0.09)
    qkv, out, want = P.normal(B, H + 2 * G, D), *(torch.empty(B, H, D, dtype=P.dtype, device=dev()) for _ in range(2))
    q, k, v, turned = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:], torch.empty(B, H, D, dtype=P.dtype, device=dev())
    angle = torch.rand(1000, D // 2, generator=P.gen, device=dev()) * 6
    rope = tman.Rope(torch.stack([angle.cos(), angle.sin()], -1).contiguous())
    ws = torch.zeros(tman.tman_attn_decode_workspace_bytes(P.cache, attn, 800), dtype=torch.uint8, device=dev())
    append = tman.bound_rope_append(P.cache, q, k, v, P.lens, turned, rope=rope)
    decode = tman.bound_attn_decode(P.cache, attn, turned, P.lens, out, 800, ws)
    s = torch.cuda.Stream()
    for _ in range(3):
        P.lens -= 1
        qkv.copy_(P.normal(*qkv.shape))
        torch.cuda.synchronize()
        append(s.cuda_stream)
        decode(s.cuda_stream)
        s.synchronize()
        pages, queries = P.k.clone(), turned.clone()
        tman.tman_rope_append(P.cache, q, k, v, P.lens, turned, rope=rope)
        tman.tman_attn_decode(P.cache, attn, turned, P.lens, want, 800, ws)
        assert torch.equal(out, want) and torch.equal(P.k, pages) and torch.equal(turned, queries)
    assert tman.tman_device_status() == 0
    with pytest.raises(tman.TmanError):
        tman.bound_attn_decode(P.cache, attn, turned[:2], P.lens, out, 800, ws)
    with pytest.raises(tman.TmanError):
        tman.bound_rope_append(P.cache, q, k, v, P.lens, None, rope=rope)


@pytest.mark.parametrize("sloped", [False, True])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("tokens", [0, 40, 600])  # single-token attention, few rows
def test_capped_scores_of_single_positions(tokens, dim, sloped):
    """A row that sees itself alone has its capped score as the logarithm of its sum: small scores as precise as large ones.

    The products are exact here (one element of query and key is not zero).  Above half the cap the score has the rounding of the
    exponential, the reciprocal and the sum, 4.3e-7 cap of at least 0.46 cap; below it some five roundings of 2^-24 and a fit of 2^-26;
    the logarithm two more: within 2^-19 in all."""
    n, cap = max(tokens, 1), 16.0
    seqs = 200 if tokens == 0 else 1
    P = Problem(dim + tokens, [n] * seqs, 4, 4, dim, 32, torch.float16, poison=0.0)
    size = torch.exp2(torch.empty(P.k.shape[:3], device=dev()).uniform_(-9, 6, generator=P.gen))
    sign = torch.where(torch.rand(P.k.shape[:3], generator=P.gen, device=dev()) < 0.5, -1.0, 1.0)
    P.k.zero_()
    P.k[..., 0] = (size * sign).half()
    attn = tman.Attn(4, 1.0, cap=cap, window=1, slopes=P.slopes() if sloped else None)
    rows = seqs * n
    q = torch.zeros(rows, 4, dim, dtype=torch.float16, device=dev())
    q[..., 0] = 1
    out, lse = torch.empty_like(q), torch.empty(rows, 4, device=dev())
    if tokens == 0:
        ws = torch.zeros(max(16, tman.tman_attn_decode_workspace_bytes(P.cache, attn, n, False)), dtype=torch.uint8, device=dev())
        tman.tman_attn_decode(P.cache, attn, q, P.lens, out, n, ws, lse=lse)
    else:
        ws = torch.zeros(max(16, tman.tman_attn_prefill_workspace_bytes(P.cache, attn, n, n)), dtype=torch.uint8, device=dev())
        tman.tman_attn_prefill(P.cache, attn, q, P.ints([0, n]), P.lens, out, n, ws, lse=lse)
    pages = P.table[:, :(n + P.page - 1) // P.page].long()
    k = P.k[pages][..., 0].double().transpose(2, 3).reshape(seqs, -1, 4)[:, :n].reshape(rows, 4)
    want = cap * torch.tanh(k / cap)
    off = ((lse.double() - want) / want).abs().max().item()
    assert off <= 2.0 ** -19, off
