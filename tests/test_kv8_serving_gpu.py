"""Plan, append and attention of an 8-bit cache one after another, as examples/serving_block.py runs them between its low-bit products:
every stage against its own plain form on what the stage before it gave, eager and as a captured graph; single tokens in a graph whose
lengths grow on the device."""
import os
import random
import sys

import pytest
import torch

import kv8_ref as ref
import paper_2511_11248_amd as tman
from attention_ref import attend
from gpu_helpers import dev
from test_kv8_attention_gpu import Problem8, within
from test_kv_plan_gpu import plain

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def state(block):
    return {n: getattr(block, n).clone() for n in ("table", "lens", "free_pages", "free_left", "q_start", "k_pages", "v_pages", "k_exps", "v_exps")}


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def check_step(block, before, more, rows):
    lens, left = before["lens"].tolist(), before["free_left"].item()
    want = plain(before["table"].tolist(), block.page, lens, more, before["free_pages"].tolist(), left, rows)
    for name, w in zip(("table", "lens", "free_left", "q_start"), (want[0], want[1], [want[2]], want[3])):
        assert getattr(block, name).tolist() == w, name
    qkv, y = block.last
    h, g, d = block.heads, block.kv_heads, block.dim
    starts, now = want[3], want[1]
    for b, n in enumerate(now):
        t = starts[b + 1] - starts[b]
        if not t:
            continue
        used = block.table[b, :-(-n // block.page)].long()
        held = []
        for pages, exps in ((block.k_pages, block.k_exps), (block.v_pages, block.v_exps)):
            x = ref.decode(pages.view(torch.uint8)[used], exps[used]).transpose(0, 1)
            held.append(x.reshape(g, -1, d)[:, :n])
        # new values are what the products gave, to half a step of a code
        v = qkv[starts[b]:starts[b + 1], h + g:].double().transpose(0, 1)
        off = (held[1][:, n - t:] - v).abs()
        most = v.abs().amax(-1, keepdim=True).amax(1, keepdim=True).clamp(min=held[1].abs().max())
        assert bool((off <= torch.maximum(v.abs() * 2.0 ** -4, most * 2.0 ** -16)).all())
        for i in sorted({0, t // 2, t - 1}):
            o, _, _, bound, _, _ = attend(qkv[starts[b] + i, :h], *held, n - t + i, 0, n - t + i + 1, block.attn.scale, 0.0, None, 0, torch.float16)
            within(y[starts[b] + i], o, bound, f"token {i} of sequence {b}")
    assert bool((y[starts[-1]:] == 0).all())


def requests(r, lens, first):
    return [r.randint(1, 90) if first else -n if n and r.random() < 0.15 else 1 if n and r.random() < 0.8 else r.choice([0, r.randint(1, 60)]) for n in lens]


@pytest.mark.parametrize("dim,pages", [(64, 200), (128, 60)])
def test_steps_of_a_server_eager_and_captured(dim, pages):
    """Twelve steps; the graph is captured once and replayed on the very states that the eager steps start from, with eager work between."""
    from serving_block import ServingBlock

    B, rows, r = 10, 400, random.Random(dim)
    block = ServingBlock(hidden=256, heads=4, kv_heads=2, dim=dim, seqs=B, most=512, page=16, pages=pages, seed=1)
    twin = ServingBlock(hidden=256, heads=4, kv_heads=2, dim=dim, seqs=B, most=512, page=16, pages=pages, seed=1)
    x = torch.zeros(rows, 256, dtype=torch.float16, device=dev())
    twin.step(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = twin.step(x)
    for name, t in state(block).items():
        getattr(twin, name).copy_(t)
    gen = torch.Generator(device=dev())
    gen.manual_seed(7)
    for step in range(12):
        more = requests(r, block.lens.tolist(), step == 0)
        before = state(block)
        block.more.copy_(torch.tensor(more, dtype=torch.int32))
        twin.more.copy_(block.more)
        x.copy_(torch.randn(rows, 256, generator=gen, device=dev()).half())
        y = block.step(x)
        assert tman.tman_device_status() == 0
        check_step(block, before, more, rows)
        graph.replay()
        torch.cuda.synchronize()
        for name, t in state(block).items():
            assert same_bits(getattr(twin, name), t), (step, name)
        assert torch.equal(out, y)


def test_single_tokens_in_a_graph_whose_lengths_grow():
    """Plan, append and single-token attention captured with lens in place: 40 replays cross pages and blocks."""
    P = Problem8(5, [1, 15, 31, 100], 4, 2, 128, 16, torch.bfloat16, extra=40)
    B, H, G, D = 4, 4, 2, 128
    ints = P.ints
    # a table with room, and the free pages
    used = sorted(set(int(p) for b, n in enumerate(P.lens_list) for p in P.table[b, :-(-n // 16)].tolist()))
    free = [p for p in range(P.k.shape[0]) if p not in used]
    table = torch.zeros(B, 12, dtype=torch.int32, device=dev())
    for b, n in enumerate(P.lens_list):
        table[b, :-(-n // 16)] = P.table[b, :-(-n // 16)]
    stack, left, lens, more = ints(free), ints([len(free)]), P.lens.clone(), ints([1] * B)
    q_start, qkv = ints([0] * (B + 1)), P.normal(B, H + 2 * G, D)
    q_out, out, lse = P.normal(B, H, D), P.normal(B, H, D), torch.zeros(B, H, device=dev())
    cache = tman.KvCache8(P.k, P.v, P.ke, P.ve, table, torch.bfloat16)
    attn = tman.Attn(H, 0.08, cap=20.0)
    ws = torch.zeros(tman.tman_attn_decode_kv8_workspace_bytes(cache, attn, 160), dtype=torch.uint8, device=dev())
    plan = tman.bound_kv_plan(table, 16, lens, more, stack, left, lens, left, q_start, n_tokens=B)
    append = tman.bound_kv8_append(cache, qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:], lens, q_out, norm=tman.HeadNorm(None, None, 1e-5))
    decode = tman.bound_attn_decode_kv8(cache, attn, q_out, lens, out, 160, ws, lse=lse)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kept = [t.clone() for t in (lens, left, table, stack, P.k, P.v, P.ke, P.ve)]
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        for call in (plan, append, decode):
            call(side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    for t, k in zip((lens, left, table, stack, P.k, P.v, P.ke, P.ve), kept):
        assert same_bits(t, k)  # capturing runs nothing
    for step in range(40):
        qkv.copy_(P.normal(B, H + 2 * G, D))
        graph.replay()
        torch.cuda.synchronize()
        assert tman.tman_device_status() == 0
        now = [n + step + 1 for n in P.lens_list]
        assert lens.tolist() == now
        for b in range(B):
            pages = table[b, :-(-now[b] // 16)].long()
            rows = [ref.decode(c[pages], e[pages]).transpose(0, 1).reshape(G, -1, D)[:, :now[b]] for c, e in ((P.k, P.ke), (P.v, P.ve))]
            o, l, _, bound, l_bound, _ = attend(q_out[b], *rows, now[b] - 1, 0, now[b], 0.08, 20.0, None, 0, torch.bfloat16)
            within(out[b], o, bound, f"step {step}, sequence {b}")
            within(lse[b], l, l_bound, f"lse, step {step}, sequence {b}")
    held = [p for b in range(B) for p in table[b, :-(-(P.lens_list[b] + 40) // 16)].tolist()]
    assert len(set(held + stack.tolist()[:left.item()])) == len(held) + left.item()


def test_chunks_and_single_calls_hold_the_same_values_where_blocks_are_whole():
    """A prompt in chunks of whole blocks leaves the same codes as in one piece; other cuts stay within what a code may be off."""
    N, G, D = 200, 2, 64
    gen = torch.Generator(device=dev())
    gen.manual_seed(3)
    kv = torch.randn(N, 2 * G, D, generator=gen, device=dev()).half()
    made = []
    for cuts in ([0, 200], [0, 64, 160, 200], [0, 7, 50, 51, 133, 200]):
        k, v = (torch.zeros(8, G, 32, D, dtype=torch.uint8, device=dev()) for _ in range(2))
        ke, ve = (torch.zeros(8, G, 2, dtype=torch.uint8, device=dev()) for _ in range(2))
        table = torch.arange(8, dtype=torch.int32, device=dev())[None].contiguous()
        cache = tman.KvCache8(k, v, ke, ve, table, torch.float16)
        for a, b in zip(cuts, cuts[1:]):
            lens, starts = (torch.tensor(x, dtype=torch.int32, device=dev()) for x in ([b], [0, b - a]))
            tman.tman_kv8_append(cache, None, kv[a:b, :G], kv[a:b, G:], lens, None, q_start=starts)
        made.append((k, v, ke, ve))
    for t, u in zip(made[0], made[1]):
        assert torch.equal(t, u)
    for c, e, c0, e0 in ((made[2][0], made[2][2], made[0][0], made[0][2]), (made[2][1], made[2][3], made[0][1], made[0][3])):
        assert torch.equal(e, e0)  # (the largest value of a block decides, whenever it came)
        x, y = ref.decode(c, e), ref.decode(c0, e0)
        # two roundings of a code that became subnormal: half a step of the power of two each
        step = torch.exp2(e.double() - 127 - 9).repeat_interleave(16, -1)[..., None]
        assert bool(((x - y).abs() <= step).all())
