"""Single tokens over an 8-bit cache whose pieces are long: lengths of some hundred thousand positions, alike and not, bounds that nothing
reaches, windows that begin inside a piece."""
import pytest
import torch

from test_kv8_attention_gpu import Problem8, check_decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,heads,kv_heads,dim,page", [([140001], 4, 4, 128, 64), ([131072, 131072], 8, 8, 128, 128), ([140001, 33000, 1, 0], 6, 3, 128, 16),
                                                          ([270000], 2, 1, 64, 256), ([70000, 65536], 4, 4, 256, 32)])
def test_long_pieces(lens, heads, kv_heads, dim, page):
    P = Problem8(dim + heads, lens, heads, kv_heads, dim, page, torch.bfloat16)
    _, ws = check_decode(P)
    check_decode(P, workspace=ws, window=65000, cap=30.0)
    check_decode(P, workspace=ws, first=[n // 3 for n in lens])


def test_long_bounds_and_short_sequences():
    P = Problem8(7, [900, 40000, 17], 8, 8, 128, 64, torch.float16)
    P.table = torch.cat([P.table, torch.full((3, 8192 - P.table.shape[1]), 2 ** 30, dtype=torch.int32, device=P.table.device)], 1).contiguous()
    P.cache = type(P.cache)(P.k, P.v, P.ke, P.ve, P.table, P.dtype)
    check_decode(P, bound_len=524288)
