"""Calls that are marshalled once hold what their pointers lead to, for as long as they are there themselves."""
import gc
import weakref

import pytest
import torch

import paper_2511_11248_amd as tman

B, H, G, D, PAGE = 2, 4, 2, 64, 16


def _tensors():
    pages = torch.zeros(8, G, PAGE, D, dtype=torch.float16)
    rows = {name: torch.zeros(B, n, D, dtype=torch.float16) for name, n in (("q", H), ("k", G), ("v", G), ("out", H))}
    ints = {name: torch.zeros(B, dtype=torch.int32) for name in ("lens", "first", "positions")}
    return dict(k_pages=pages, v_pages=pages.clone(), table=torch.zeros(B, 4, dtype=torch.int32), **rows, **ints,
                q_start=torch.arange(B + 1, dtype=torch.int32), cos_sin=torch.zeros(8, D // 2, 2), slopes=torch.zeros(H),
                weights=torch.zeros(8, G, PAGE), lse=torch.zeros(B, H), workspace=torch.zeros(1 << 20, dtype=torch.uint8))


def _append(t):
    cache = tman.KvCache(t["k_pages"], t["v_pages"], t["table"])
    return tman.bound_rope_append(cache, t["q"], t["k"], t["v"], t["lens"], t["out"], rope=tman.Rope(t["cos_sin"]), positions=t["positions"],
                                  q_start=t["q_start"], weights=t["weights"])


def _decode(t):
    cache = tman.KvCache(t["k_pages"], t["v_pages"], t["table"])
    return tman.bound_attn_decode(cache, tman.Attn(H, 1.0, slopes=t["slopes"]), t["q"], t["lens"], t["out"], 64, t["workspace"],
                                  first=t["first"], lse=t["lse"], weights=t["weights"])


@pytest.mark.parametrize("bind,used", [
    (_append, "k_pages v_pages table q k v lens out cos_sin positions q_start weights"),
    (_decode, "k_pages v_pages table slopes q lens out workspace first lse weights"),
])
def test_a_bound_call_keeps_its_tensors(bind, used):
    t = _tensors()
    call = bind(t)
    alive = {name: weakref.ref(t[name]) for name in used.split()}
    del t
    gc.collect()
    assert [name for name, ref in alive.items() if ref() is None] == []
    del call
    gc.collect()
    assert [name for name, ref in alive.items() if ref() is not None] == []


def test_a_single_token_has_no_stride():
    """Where there is one token the distance to the next says nothing: k as a column of a fused matrix beside v of its own is taken, and so
    is any distance that torch keeps for a dimension of one."""
    cache = tman.KvCache(torch.zeros(8, G, PAGE, D, dtype=torch.float16), torch.zeros(8, G, PAGE, D, dtype=torch.float16),
                         torch.zeros(1, 4, dtype=torch.int32))
    lens = torch.zeros(1, dtype=torch.int32)
    fused = torch.zeros(1, H + 2 * G, D, dtype=torch.float16)
    tman.bound_rope_append(cache, fused[:, :H], fused[:, H:H + G], torch.zeros(1, G, D, dtype=torch.float16), lens, fused[:, :H])
    odd = torch.zeros(1030, dtype=torch.float16).as_strided((1, H, D), (1030, D, 1))
    with pytest.raises(tman.TmanError) as e:
        tman.tman_attn_decode(cache, tman.Attn(H, 1.0), odd, lens, odd.clone(), 64, None, stream=0)
    assert e.value.status == -5  # the workspace alone is missing
