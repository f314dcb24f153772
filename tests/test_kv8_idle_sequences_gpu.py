"""Prompts over an 8-bit cache beside sequences that have no token in the call: nothing of those is read, copied or reported, as in the call
over a 16-bit cache."""
import pytest
import torch

import paper_2511_11248_amd as tman
from gpu_helpers import dev
from test_kv8_attention_gpu import Problem8, check_prefill

pytestmark = pytest.mark.gpu
TICKETS = 16384  # bytes in front of a workspace, zeroed by the caller


def problem(dim=64, kv_heads=8):
    """One prompt of 1100 tokens behind 300 positions, among seven idle sequences."""
    return Problem8(dim, [700, 1500, 0, 1400, 33, 1900, 1, 1200], 4 * kv_heads, kv_heads, dim, 32, torch.float16), [0, 0, 0, 1100, 0, 0, 0, 0]


@pytest.mark.parametrize("window", [0, 40, 1000])
def test_idle_sequences_may_have_no_pages_and_any_length(window):
    P, new = problem()
    idle = [b for b, t in enumerate(new) if not t]
    P.table[idle] = 2 ** 30
    P.lens_list = [n if t else 0 for n, t in zip(P.lens_list, new)]  # (the plain form looks up no pages of theirs)
    # (the last ones are longer than the bound, one beyond any table)
    P.lens[5], P.lens[7] = 2 ** 31 - 1, 5000
    check_prefill(P, new, window=window, bound_len=2100, sample=range(0, 1100, 97))


@pytest.mark.parametrize("window", [0, 40, 1000])
def test_idle_sequences_are_not_copied(window):
    """One workgroup a row tile, so that the workspace holds the copy, its table, and nothing else behind the tickets."""
    P, new = problem()
    G, D, bound = P.kv_heads, P.dim, 2100
    attn = tman.Attn(P.heads, D ** -0.5, window=window)
    need = tman.tman_attn_prefill_kv8_workspace_bytes(P.cache, attn, sum(new) + 3, bound)
    ws = torch.full((need,), 0xa5, dtype=torch.uint8, device=dev())
    ws[:TICKETS] = 0
    check_prefill(P, new, window=window, bound_len=bound, workspace=ws, sample=[0, 99, 700])
    seen = 1400 if not window else min(1400, 1100 + window)  # positions that some token sees, and what fills their tiles of 64
    wrote = int((ws[TICKETS:] != 0xa5).sum())
    assert 0 < wrote <= 2 * (seen + 128) * G * D * 2 + 8 * (-(-bound // P.page)) * 4


def test_offsets_beyond_the_tokens_are_cut_alike_for_copy_and_attention():
    """q_start names more tokens than the call has: the sequence's last positions are those that the call has."""
    P, new = problem()
    N, n, bound = 1100, 1400, 2100
    attn = tman.Attn(P.heads, P.dim ** -0.5, window=50)
    q = P.normal(N, P.heads, P.dim)
    outs = []
    for last in (N, N + 500):
        ws = torch.full((tman.tman_attn_prefill_kv8_workspace_bytes(P.cache, attn, N, bound),), 0xff, dtype=torch.uint8, device=dev())
        ws[:TICKETS] = 0
        out = torch.empty_like(q)
        tman.tman_attn_prefill_kv8(P.cache, attn, q, P.ints([0, 0, 0, 0, last, last, last, last, last]), P.lens, out, bound, ws)
        outs.append(out)
    tman.tman_device_status()
    assert torch.equal(*outs) and bool(torch.isfinite(outs[0]).all())
