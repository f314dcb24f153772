"""The attention block of a decoder that serves requests as they come, on the library alone: pages planned on the GPU, fused QKV product
with low-bit weights, norms of heads, rotary positions and append to a cache held in 8 bits, attention, output product.  A step takes
whatever comes: prompts, chunks of them, single tokens, sequences that end; it is one captured graph for a given number of rows.

    python examples/serving_block.py [--seqs 16] [--steps 60] [--pages 400]

Weights and requests are random; what is printed is the time of a step and how the pages were used.
"""
from __future__ import annotations

import argparse
import os
import random
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from attention_block import Linear, tman  # noqa: E402


class ServingBlock:
    def __init__(self, hidden=1024, heads=8, kv_heads=2, dim=128, bits=4, group=64, seqs=16, most=1024, page=32, pages=400, seed=0,
                 device="cuda"):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.hidden, self.heads, self.kv_heads, self.dim, self.seqs, self.most, self.page = hidden, heads, kv_heads, dim, seqs, most, page
        self.qkv = Linear((heads + 2 * kv_heads) * dim, hidden, bits, group, gen)
        self.out = Linear(hidden, heads * dim, bits, group, gen)
        self.k_pages, self.v_pages = (torch.zeros(pages, kv_heads, page, dim, dtype=torch.float8_e4m3fn, device=device) for _ in range(2))
        self.k_exps, self.v_exps = (torch.zeros(pages, kv_heads, page // 16, dtype=torch.uint8, device=device) for _ in range(2))
        ints = lambda *n: torch.zeros(*n, dtype=torch.int32, device=device)  # noqa: E731
        self.table, self.lens, self.more, self.q_start = ints(seqs, most // page), ints(seqs), ints(seqs), ints(seqs + 1)
        self.free_pages = torch.randperm(pages, generator=gen, device=device).to(torch.int32)
        self.free_left = torch.tensor([pages], dtype=torch.int32, device=device)
        self.cache = tman.KvCache8(self.k_pages, self.v_pages, self.k_exps, self.v_exps, self.table, torch.float16)
        self.norm = tman.HeadNorm(1 + 0.1 * torch.randn(dim, generator=gen, device=device), 1 + 0.1 * torch.randn(dim, generator=gen, device=device), 1e-6)
        at = torch.arange(most, dtype=torch.float64, device=device)
        angle = at[:, None] * 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=device) / dim)
        self.rope = tman.Rope(torch.stack([angle.cos(), angle.sin()], -1).float().contiguous())
        self.attn = tman.Attn(heads, dim ** -0.5)
        self.workspaces = {}

    def _workspaces(self, rows):
        """Of the plan and of the attention, zeroed once, and the places of the tokens."""
        if rows not in self.workspaces:
            needs = (tman.tman_kv_plan_workspace_bytes(self.seqs, rows), tman.tman_attn_prefill_kv8_workspace_bytes(self.cache, self.attn, rows, self.most))
            self.workspaces[rows] = [*(torch.zeros(max(n, 16), dtype=torch.uint8, device=self.lens.device) for n in needs),
                                     *(torch.zeros(rows, dtype=torch.int32, device=self.lens.device) for _ in range(2))]
        return self.workspaces[rows]

    def step(self, x):
        """x [rows, hidden]: the tokens that self.more asks for, sequence after sequence.  Those of sequences that have to wait are left out, and
        the others move up: returns [rows, hidden] in the order of q_start, whose rows behind the last token are padding.  lens, q_start, the
        page table and the free pages are up to date afterwards."""
        rows, h, g, d = x.shape[0], self.heads, self.kv_heads, self.dim
        plan_space, space, positions, owners = self._workspaces(rows)
        asked, before = self.more.clamp(min=0), self.lens.clone()
        tman.tman_kv_plan(self.table, self.page, self.lens, self.more, self.free_pages, self.free_left, self.lens, self.free_left, self.q_start,
                          positions=positions, owners=owners, workspace=plan_space, n_tokens=rows)
        owner = owners.clamp(min=0).long()
        source = (asked.cumsum(0) - asked)[owner] + positions - before[owner]
        x = x[source.clamp(0, rows - 1)]
        qkv = self.qkv(x).view(rows, h + 2 * g, d)
        q, k, v = qkv[:, :h], qkv[:, h:h + g], qkv[:, h + g:]
        tman.tman_kv8_append(self.cache, q, k, v, self.lens, q, norm=self.norm, rope=self.rope, q_start=self.q_start)
        y = torch.zeros(rows, h, d, dtype=torch.float16, device=x.device)
        tman.tman_attn_prefill_kv8(self.cache, self.attn, q, self.q_start, self.lens, y, self.most, space)
        self.last = qkv, y  # what the append and the attention took and gave
        return self.out(y.view(rows, -1))


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("seqs", 16), ("steps", 60), ("pages", 400)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    block, r, rows = ServingBlock(seqs=a.seqs, pages=a.pages), random.Random(0), 256
    x = torch.randn(rows, block.hidden, device="cuda").half()
    block.step(x)  # (nothing is asked for yet)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = block.step(x)
    spent, tokens, waiting = 0.0, 0, 0
    for _ in range(a.steps):
        lens = block.lens.tolist()  # (a server keeps its own count)
        more = [-n if n and r.random() < 0.05 else 1 if n else r.choice([0, r.randint(1, 100)]) for n in lens]
        block.more.copy_(torch.tensor(more, dtype=torch.int32))
        x.copy_(torch.randn(rows, block.hidden, device="cuda").half())
        torch.cuda.synchronize()
        t = time.perf_counter()
        graph.replay()
        torch.cuda.synchronize()
        spent += time.perf_counter() - t
        starts = block.q_start.tolist()
        tokens += starts[-1]
        waiting += sum(m > 0 and starts[b + 1] == starts[b] for b, m in enumerate(more))
        assert bool(y[:starts[-1]].isfinite().all())
    print(f"{a.steps} steps, {tokens} tokens, {waiting} times a sequence had to wait for pages: {1e3 * spent / a.steps:.3f} ms a step; lengths "
          f"{block.lens.tolist()}, {block.free_left.item()} of {a.pages} pages free")
    assert tman.tman_device_status() == 0


if __name__ == "__main__":
    main()
