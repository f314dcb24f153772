"""The serving example's rows: a sequence that has to wait for pages keeps its rows of the input, and those behind it keep theirs."""
import os
import sys

import pytest
import torch

import paper_2511_11248_amd as tman
from gpu_helpers import dev

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
HIDDEN, ROWS = 256, 64


def block(pages):
    from serving_block import ServingBlock

    return ServingBlock(hidden=HIDDEN, heads=4, kv_heads=2, dim=64, seqs=4, most=128, page=16, pages=pages, seed=3)


def step(b, more, x):
    b.more.copy_(torch.tensor(more, dtype=torch.int32))
    y = b.step(x).clone()
    assert tman.tman_device_status() == 0
    return y, b.q_start.tolist()


@pytest.mark.parametrize("captured", [False, True])
def test_rows_behind_a_sequence_that_waits(captured):
    """Four pages: a prompt of 40 in the middle is refused, the single tokens around it fit into the pages that their sequences have."""
    gen = torch.Generator(device=dev())
    gen.manual_seed(9)
    first, x = (torch.randn(ROWS, HIDDEN, generator=gen, device=dev()).half() for _ in range(2))
    waits, never = block(4), block(4)
    rows = first.clone()
    run = {}
    if captured:
        for b in (waits, never):
            b.step(rows)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out = b.step(rows)
            run[id(b)] = graph, out

    def go(b, more, data):
        if not captured:
            return step(b, more, data)
        b.more.copy_(torch.tensor(more, dtype=torch.int32))
        rows.copy_(data)
        graph, out = run[id(b)]
        graph.replay()
        torch.cuda.synchronize()
        assert tman.tman_device_status() == 0
        return out.clone(), b.q_start.tolist()

    for b in (waits, never):
        _, starts = go(b, [5, 0, 7, 17], first)
        assert starts == [0, 5, 5, 12, 29]
    for k in range(3):  # (the same again: replays, and sequences that go on)
        y, starts = go(waits, [1, 40, 1, 2], x)
        assert starts == [0, 1, 1, 2, 4]
        # as if the prompt had not asked: its forty rows are not there
        z, starts = go(never, [1, 0, 1, 2], torch.cat([x[:1], x[41:44], x[:ROWS - 4]]))
        assert starts == [0, 1, 1, 2, 4]
        assert torch.equal(y[:4], z[:4])
        for n in ("lens", "table", "free_left"):
            assert torch.equal(getattr(waits, n), getattr(never, n)), n
        held = waits.table[3, :2].long()
        assert torch.equal(waits.v_pages.view(torch.uint8)[held], never.v_pages.view(torch.uint8)[held])


def test_rows_of_a_step_that_everybody_gets():
    gen = torch.Generator(device=dev())
    gen.manual_seed(10)
    x = torch.randn(ROWS, HIDDEN, generator=gen, device=dev()).half()
    b = block(40)
    values = lambda x: b.qkv(x).view(ROWS, 8, 64)[:, 6:]  # noqa: E731
    _, starts = step(b, [5, 0, 7, 17], x)
    assert starts == [0, 5, 5, 12, 29]
    assert torch.equal(b.last[0][:29, 6:], values(x)[:29])
    _, starts = step(b, [-5, 3, 1, 1], x)
    assert starts == [0, 0, 3, 4, 5]
    assert torch.equal(b.last[0][:5, 6:], values(x)[:5])
