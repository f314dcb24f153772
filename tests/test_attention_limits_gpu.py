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
