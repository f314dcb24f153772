"""Sizes, masks and numbers at which the key-value cache's operators are at their limits.  The references and bounds are those of
test_attention_gpu.py where nothing else is said."""
import pytest
import torch

import paper_2511_11248_amd as tman
from attention_ref import attend, gather
from gpu_helpers import dev
from test_attention_gpu import Problem, check_prefill, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,heads,kv_heads,dim", [(1000, 1, 1, 256), (130, 8, 8, 128), (256, 4, 2, 128)])
def test_a_prompt_workspace_of_a_longer_bound_serves_a_shorter_prompt(tokens, heads, kv_heads, dim):
    P = Problem(tokens, [1990], heads, kv_heads, dim, 32, torch.float16)
    need = tman.tman_attn_prefill_workspace_bytes(P.cache, tman.Attn(heads, 1.0), tokens, 2100)
    ws = torch.zeros(need, dtype=torch.uint8, device=dev())
    for bound in (2100, 2000, 2048, 1990):
        check_prefill(P, [tokens], rows=8, workspace=ws, bound_len=bound)


def test_new_lengths_in_the_place_of_the_old_ones():
    """Many heads a sequence, so that some are chosen for after others are done."""
    lens, keep, recent, G = [3000, 40, 700, 2500], 300, 20, 64
    P = Problem(61, lens, G, G, 64, 64, torch.float16, spare_pages=2 * 4 * 5)
    w = torch.rand(P.k.shape[:3], generator=P.gen, device=dev())
    spare = list(P.spare)
    tables = [P.ints([[spare.pop() for _ in range(5)] for _ in range(4)]) for _ in range(2)]
    results = []
    for table, own in zip(tables, (False, True)):
        old = P.lens.clone()
        new = old if own else torch.empty_like(old)
        kept = torch.full((4, G, keep), 99, dtype=torch.int32, device=dev())
        tman.tman_kv_evict(P.cache, w, old, keep, recent, table, new, kept, 3000)
        assert tman.tman_device_status() == 0
        assert new.tolist() == [min(n, keep) for n in lens]
        moved = [pages[table.long()].transpose(1, 2).flatten(2, 3) for pages in (P.k, P.v, w)]  # [sequence, head, position, ...]
        moved = [x[b, :, :min(lens[b], keep)] for x in moved for b in range(4)]
        results.append([kept] + moved)
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("tokens", [1, 5, 150])  # single-token attention, few rows, many
def test_many_small_probabilities_add_up(tokens, dim):
    """Four positions of large weight, one for every wave that takes positions of its own, whose values are zero, and 131068 of exp(-17.6875) =
    2^-25.5 of it each, whose values are one: together they are the result, 6.8e-4.

    Half precision with the largest probability at one has nothing for them.  With a reference 2^7 lower at least they have steps of 2^-24 at
    2^-18.5, so 2^-6.5 of a probability is lost at most; beside that, the rounding of the result (2^-11), what the lanes that hold the four
    lose of the small ones in 32-bit sums (a quarter of 6.8e-4), and some 2^-11 of the sums' roundings: within 2^-6 of the result."""
    n, seqs, peaks = 131072, 256, [0, 32, 64, 96]
    P = Problem(71, [n], 1, 1, dim, 256, torch.float16, poison=0.0)
    P.k.zero_()
    P.v.fill_(1.0)
    for j in peaks:
        page, slot = P.row(0, j)
        P.k[page, 0, slot, 0], P.v[page, 0, slot] = 17.6875, 0.0
    # all sequences read the same pages: a batch that fills the chip, so that rows are not cut in pieces
    cache, lens = tman.KvCache(P.k, P.v, P.table.repeat(seqs, 1)), P.lens.repeat(seqs)
    rows = seqs * tokens
    q = torch.zeros(rows, 1, dim, dtype=torch.float16, device=dev())
    q[..., 0] = 1
    out = torch.empty_like(q)
    attn = tman.Attn(1, 1.0)
    if tokens == 1:
        ws = torch.zeros(tman.tman_attn_decode_workspace_bytes(cache, attn, n), dtype=torch.uint8, device=dev())
        tman.tman_attn_decode(cache, attn, q, lens, out, n, ws)
    else:
        ws = torch.zeros(max(16, tman.tman_attn_prefill_workspace_bytes(cache, attn, rows, n)), dtype=torch.uint8, device=dev())
        starts = torch.arange(0, rows + 1, tokens, dtype=torch.int32, device=dev())
        tman.tman_attn_prefill(cache, attn, q, starts, lens, out, n, ws)
    assert tman.tman_device_status() == 0
    seen = n - tokens + 1 + torch.arange(tokens, dtype=torch.float64, device=dev())
    small = (seen - 4) * torch.tensor(-17.6875, dtype=torch.float64).exp().item()
    want = (small / (4 + small)).repeat(seqs)[:, None, None]
    off = ((out.double() - want) / want).abs().max().item()
    assert off <= 2.0 ** -6, off


@pytest.mark.parametrize("cap", [300.0, 1e4, 1e7])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("tokens", [1, 30, 400])  # single-token attention, few rows, many
def test_large_caps_leave_small_scores_alone(tokens, dim, cap):
    """cap tanh(s / cap) with a relative error of 2^-20, so no further off than the products are (a score of `dim` products: (dim + 8) 2^-24 of the
    sum of their sizes): the bound of scores that are not capped holds."""
    n = 5000
    P = Problem(73 + tokens, [n], 4, 2, dim, 64, torch.float16)
    q = P.normal(tokens, 4, dim)
    out, lse = torch.empty_like(q), torch.empty(tokens, 4, device=dev())
    attn, scale = tman.Attn(4, dim ** -0.5, cap=cap), dim ** -0.5
    if tokens == 1:
        ws = torch.zeros(tman.tman_attn_decode_workspace_bytes(P.cache, attn, n), dtype=torch.uint8, device=dev())
        tman.tman_attn_decode(P.cache, attn, q, P.lens, out, n, ws, lse=lse)
    else:
        ws = torch.zeros(max(16, tman.tman_attn_prefill_workspace_bytes(P.cache, attn, tokens, n)), dtype=torch.uint8, device=dev())
        tman.tman_attn_prefill(P.cache, attn, q, P.ints([0, tokens]), P.lens, out, n, ws, lse=lse)
    k, v = gather(P.k, P.table, 0, n), gather(P.v, P.table, 0, n)
    for i in sorted({0, tokens // 3, tokens - 1}):
        at = n - tokens + i
        o, l, *_ = attend(q[i], k, v, at, 0, at + 1, scale, cap, None, 0, P.dtype)
        *_, bound, l_bound, _ = attend(q[i], k, v, at, 0, at + 1, scale, 0.0, None, 0, P.dtype)
        within(out[i], o, bound, f"out, token {i}")
        within(lse[i], l, l_bound, f"lse, token {i}")


@pytest.mark.parametrize("tokens", [1, 30, 400])
def test_a_cap_of_next_to_nothing_makes_all_scores_alike(tokens):
    """Also the score of a product of zero: the result is the mean of the values."""
    n, H, D = 3000, 2, 64
    P = Problem(75, [n], H, 1, D, 64, torch.float16)
    q = P.normal(tokens, H, D)
    q[:, 0] = 0
    out = torch.empty_like(q)
    attn = tman.Attn(H, 1.0, cap=1e-42)
    ws = torch.zeros(32 << 20, dtype=torch.uint8, device=dev())
    if tokens == 1:
        tman.tman_attn_decode(P.cache, attn, q, P.lens, out, n, ws)
    else:
        tman.tman_attn_prefill(P.cache, attn, q, P.ints([0, tokens]), P.lens, out, n, ws)
    k, v = gather(P.k, P.table, 0, n), gather(P.v, P.table, 0, n)
    for i in sorted({0, tokens - 1}):
        at = n - tokens + i
        o, _, _, bound, _, _ = attend(torch.zeros_like(q[i]), k, v, at, 0, at + 1, 1.0, 0.0, None, 0, P.dtype)
        within(out[i], o, bound, f"token {i}")


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_capped_scores_of_single_positions_among_many_rows(dim):
    """What the kernel for many rows promises of a row that sees itself alone: its score to 4.3e-7 cap.

    Beside it the reference below the score, the exponential's argument, the sum's logarithm (about 7) and their sum are rounded in units of
    powers of two, 2^-21 each with the logarithm's own error: less than 2^-19 together; and lse once, 2^-24 of itself.  The bound of 2100
    positions keeps the kernel for few rows out of it."""
    n, cap, heads = 600, 16.0, 4
    P = Problem(77 + dim, [n], heads, heads, dim, 32, torch.float16, poison=0.0)
    size = torch.exp2(torch.empty(P.k.shape[:3], device=dev()).uniform_(-9, 6, generator=P.gen))
    sign = torch.where(torch.rand(P.k.shape[:3], generator=P.gen, device=dev()) < 0.5, -1.0, 1.0)
    P.k.zero_()
    P.k[..., 0] = (size * sign).half()
    attn = tman.Attn(heads, 1.0, cap=cap, window=1)
    q = torch.zeros(n, heads, dim, dtype=torch.float16, device=dev())
    q[..., 0] = 1
    out, lse = torch.empty_like(q), torch.empty(n, heads, device=dev())
    ws = torch.zeros(max(16, tman.tman_attn_prefill_workspace_bytes(P.cache, attn, n, 2100)), dtype=torch.uint8, device=dev())
    tman.tman_attn_prefill(P.cache, attn, q, P.ints([0, n]), P.lens, out, 2100, ws, lse=lse)
    assert tman.tman_device_status() == 0
    k = gather(P.k, P.table, 0, n)[..., 0].t()
    want = cap * torch.tanh(k / cap)
    within(lse, want, 4.3e-7 * cap + 2.0 ** -19 + 2.0 ** -24 * want.abs(), "lse")
    assert torch.equal(out, gather(P.v, P.table, 0, n).transpose(0, 1).to(out.dtype))  # the probability of a single position is one


def test_one_long_chunk_among_sequences_of_one_token_or_none():
    """The choice of a kernel goes by the average: here it falls on the one for few rows."""
    new = [300] + [b % 2 for b in range(63)]
    P = Problem(79, [5000] + [1 + 40 * b for b in range(63)], 8, 2, 64, 32, torch.float16)
    check_prefill(P, new, rows=20)
    check_prefill(P, new, rows=20, cap=20.0, sloped=True, window=700)
