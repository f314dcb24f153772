"""Sizes at which the key-value cache's operators change what they do, as the host sees them: workspaces and refusals."""
import pytest

from paper_2511_11248_amd import attention as at
from test_attention_abi_cpu import ALIGN, FAKE, SHAPE, _attn, _cache, _evict

BOUNDS = (1, 31, 32, 255, 256, 257, 500, 1000, 1500, 2000, 2047, 2048, 2049, 2100, 2500, 3000, 4095, 4096, 4097, 8192, 16384, 40000, 131072, 1 << 20)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kv_heads,heads,seqs", [(1, 1, 1), (2, 4, 1), (8, 32, 1), (1, 16, 1), (4, 4, 3), (2, 14, 8), (8, 8, 64), (32, 32, 300)])
def test_a_prompt_workspace_for_a_longer_bound_serves_shorter_ones(dim, kv_heads, heads, seqs):
    """For every number of tokens, those included at which another kernel takes over."""
    L = at._load()
    c, a = _cache(kv_heads=kv_heads, n_seqs=seqs, max_pages=1 << 20, dim=dim), _attn(heads=heads)
    for tokens in (1, 2, 5, 9, 33, 64, 65, 130, 200, 256, 257, 512, 700, 1000, 1024, 1500, 2048, 3001, 8192):
        need = [L.tman_attn_prefill_workspace_bytes(c, a, tokens, n) for n in BOUNDS]
        assert need == sorted(need), (tokens, need)


def test_new_lengths_lie_in_the_place_of_the_old_ones_or_apart():
    L, c = at._load(), _cache(n_seqs=3)
    lens = FAKE + 64
    for off in (-8, -4, 4, 8):
        assert _evict(L, c, lens=lens, new=lens + off) == SHAPE
    for off in (-12, 0, 12):
        assert _evict(L, c, lens=lens, new=lens + off, w=FAKE + 4) == ALIGN  # not refused for where they lie


def test_more_is_not_kept_than_positions_can_be_numbered():
    L, c = at._load(), _cache(page=1024)
    for keep in ((1 << 30) + 1, (1 << 31) - 1025, (1 << 31) - 1):
        assert _evict(L, c, keep=keep, pages=1 << 22) == SHAPE
    assert _evict(L, c, keep=1 << 30, pages=1 << 22, w=FAKE + 4) == ALIGN  # not refused for its size
