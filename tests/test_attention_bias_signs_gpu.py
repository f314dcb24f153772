"""Distance biases of any sign: prompts whose scores fall, rise or stay with the distance, heads of one key-value head that differ in it, over
16-bit and 8-bit caches, in one piece and in several."""
import pytest
import torch

import test_attention_gpu as full
import test_kv8_attention_gpu as codes
from gpu_helpers import dev

pytestmark = pytest.mark.gpu
SIGNS = {"negative": [-1, -1, -1, -1], "mixed": [-1, 1, 0, 1], "first positive": [1, -1, 0, -1], "zero": [0, 0, 0, 0]}


@pytest.mark.parametrize("kind", [full, codes])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("signs", list(SIGNS))
@pytest.mark.parametrize("how", ["causal", "prefix", "window", "capped", "pieces", "few"])
def test_biases_of_any_sign(kind, dim, signs, how):
    lens, new = {"pieces": ([9000], [600]), "few": ([700, 40], [5, 40])}.get(how, ([1500, 333], [1500, 333]))
    P = (full.Problem if kind is full else codes.Problem8)(dim + len(signs), lens, 4, 1, dim, 32, torch.bfloat16)
    size = torch.tensor([0.02, 0.3, 0.1, 0.004], device=dev()) * torch.tensor(SIGNS[signs], device=dev())
    P.slopes = lambda: size.float().contiguous()
    end = [max(i + 1, n * 3 // 4) for n, t in zip(lens, new) for i in range(n - t, n)] if how == "prefix" else None
    kind.check_prefill(P, new, end=end, window=200 if how == "window" else 0, cap=20.0 if how == "capped" else 0.0, sloped=True,
                       **(dict(rows=8) if kind is full else dict(sample=[0, 63, 127, 128, 599, 1111])))
