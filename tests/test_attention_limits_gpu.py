"""Sizes, masks and numbers at which the key-value cache's operators are at their limits.  The references and bounds are those of
test_attention_gpu.py where nothing else is said."""
import pytest
import torch

import paper_2511_11248_amd as tman
from gpu_helpers import dev
from test_attention_gpu import Problem, check_prefill

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
