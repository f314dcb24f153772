"""The operators of the key-value cache together with the low-bit products, as examples/attention_block.py runs them: prompts, steps,
an eviction, steps; every stage against its own 64-bit form on what the stage before it gave."""
import os
import sys

import pytest
import torch

import oracle
import paper_2511_11248_amd as tman
from attention_ref import attend, gather
from gpu_helpers import TOL, dev

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def _product(linear, x, y):
    s = linear.shape
    want = oracle.matmul(*(t.cpu().numpy() for t in (linear.codes, linear.scales, linear.zeros, x)), s.bits, s.group)
    assert oracle.row_relative_error(y.cpu().numpy(), want).max() <= TOL


def _check(block, x, y, tokens):
    """tokens: (row, sequence, position in its cache) of the rows that are compared"""
    q, got = block.last
    _product(block.out, got.reshape(x.shape[0], -1), y)
    cache = block.caches[0]
    for n, b, at in tokens:
        k, v = gather(block.k_pages, cache.page_table, b, at + 1), gather(block.v_pages, cache.page_table, b, at + 1)
        out, _, _, bound, _, _ = attend(q[n], k, v, at, 0, at + 1, block.attn.scale, block.attn.cap, None, 0, torch.float16)
        assert bool(((got[n].double() - out).abs() <= bound).all()), (n, b, at)


def test_prompts_steps_eviction(oracle_lib):
    from attention_block import AttentionBlock

    B, new, budget, recent = 3, [90, 1, 57], 48, 10
    block = AttentionBlock(hidden=256, heads=4, kv_heads=2, dim=64, seqs=B, most=128, page=16, budget=budget, recent=recent, seed=3)
    starts = [sum(new[:b]) for b in range(B + 1)]
    gen = torch.Generator(device=dev())
    gen.manual_seed(5)
    rand = lambda n: torch.randn(n, 256, generator=gen, device=dev()).half()  # noqa: E731
    x = rand(starts[-1])
    y = block.prompt(x, starts, new)
    _check(block, x, y, [(starts[b] + i, b, i) for b in range(B) for i in sorted({0, new[b] // 2, new[b] - 1})])
    lens = list(new)
    for _ in range(3):
        x = rand(B)
        y = block.step(x)
        lens = [n + 1 for n in lens]
        assert block.lens.tolist() == lens
        _check(block, x, y, [(b, b, lens[b] - 1) for b in range(B)])
    before = [(gather(block.k_pages, block.caches[0].page_table, b, lens[b]), gather(block.weights, block.caches[0].page_table, b, lens[b])) for b in range(B)]
    block.make_room()
    assert block.lens.tolist() == [min(n, budget) for n in lens]
    for b in range(B):
        n = min(lens[b], budget)
        k, w = gather(block.k_pages, block.caches[0].page_table, b, n), gather(block.weights, block.caches[0].page_table, b, n)
        for g in range(2):
            kept = block.kept[b, g, :n].long()
            assert torch.equal(k[g], before[b][0][g][kept]) and torch.equal(w[g], before[b][1][g][kept])
            if lens[b] > budget:
                others = sorted(range(lens[b] - recent), key=lambda j: (-float(before[b][1][g][j]), j))[:budget - recent]
                assert kept.tolist() == sorted(others) + list(range(lens[b] - recent, lens[b]))
    lens = block.lens.tolist()
    x = rand(B)
    y = block.step(x)
    _check(block, x, y, [(b, b, lens[b]) for b in range(B)])
    # the next prompt of a conversation that has been thinned out: a few tokens behind what was kept
    lens, new = block.lens.tolist(), [4, 0, 7]
    starts = [0, 4, 4, 11]
    x = rand(11)
    y = block.prompt(x, starts, new)
    _check(block, x, y, [(starts[b] + i, b, lens[b] + i) for b in (0, 2) for i in range(new[b])])
    assert tman.tman_device_status() == 0
