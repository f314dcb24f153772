"""The attention block of a decoder with low-bit weights, on the library alone: fused QKV product, rotary positions and append to a
paged cache, attention, output product; prompts, single tokens, and eviction when the cache has reached its budget.

    python examples/attention_block.py [--seqs 4] [--prompt 300] [--steps 40] [--budget 256] [--recent 64]

Weights are random codes with random scales and zeros; what is printed is times and how much of the cache stayed.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2511_11248_amd as tman  # noqa: E402


class Linear:
    """A packed low-bit matrix [out, features]; x fp16 [tokens, features] -> y fp16 [tokens, out]."""

    def __init__(self, out: int, features: int, bits: int, group: int, gen):
        device = gen.device
        self.shape = tman.Shape(out, features, bits, group)
        self.codes = torch.randint(1 << bits, (out, features), dtype=torch.uint8, generator=gen, device=device)
        step = features ** -0.5 * 4 / (1 << bits)
        self.scales = (step * (0.5 + torch.rand(out, features // group, generator=gen, device=device))).half()
        self.zeros = ((1 << bits) / 2 + torch.rand(out, features // group, generator=gen, device=device) - 1).half()
        self.packed = torch.empty(tman.tman_packed_bytes(self.shape), dtype=torch.uint8, device=device)
        tman.tman_pack_weights(self.shape, self.codes, self.scales, self.zeros, self.packed)
        need = max(tman.tman_mpgemm_workspace_bytes(self.shape, n) for n in (1, 32))
        self.workspace = torch.zeros(max(need, 16), dtype=torch.uint8, device=device)

    def __call__(self, x):
        y = torch.empty(x.shape[0], self.shape.M, dtype=torch.float16, device=x.device)
        tman.tman_mpgemm(self.shape, self.packed, x, x.shape[0], y, self.workspace)
        return y


class AttentionBlock:
    def __init__(self, hidden=1024, heads=8, kv_heads=2, dim=128, bits=4, group=64, cap=50.0, seqs=4, most=1024, page=32,
                 budget=256, recent=64, seed=0, device="cuda"):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.seqs, self.most, self.budget, self.recent = heads, kv_heads, dim, seqs, most, budget, recent
        self.qkv = Linear((heads + 2 * kv_heads) * dim, hidden, bits, group, gen)
        self.out = Linear(hidden, heads * dim, bits, group, gen)
        # the pool: two sets of pages, the one in use and the one that an eviction fills
        pages = (most + page - 1) // page
        shape = (2 * seqs * pages, kv_heads, page, dim)
        self.k_pages, self.v_pages = (torch.zeros(shape, dtype=torch.float16, device=device) for _ in range(2))
        self.weights = torch.zeros(shape[:3], dtype=torch.float32, device=device)
        tables = torch.randperm(2 * seqs * pages, generator=gen, device=device).to(torch.int32).view(2, seqs, pages)
        self.caches = [tman.KvCache(self.k_pages, self.v_pages, t.contiguous()) for t in tables]
        self.lens = torch.zeros(seqs, dtype=torch.int32, device=device)
        self.positions = torch.zeros(seqs, dtype=torch.int32, device=device)  # of the next token, which eviction does not change
        self.longest = 0
        # angles and scores
        at = torch.arange(64 * most, dtype=torch.float64, device=device)
        freq = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=device) / dim)
        angle = at[:, None] * freq
        self.rope = tman.Rope(torch.stack([angle.cos(), angle.sin()], -1).float().contiguous())
        self.attn = tman.Attn(heads, dim ** -0.5, cap=cap)
        # one workspace for decoding and prompts, zeroed once
        need = max(tman.tman_attn_decode_workspace_bytes(self.caches[0], self.attn, most, True),
                   max(tman.tman_attn_prefill_workspace_bytes(self.caches[0], self.attn, n, most) for n in (1, seqs, 128, most)))
        self.workspace = torch.zeros(need, dtype=torch.uint8, device=device)
        self.kept = torch.empty(seqs, kv_heads, budget, dtype=torch.int32, device=device)

    def _split(self, x):
        h, g, d = self.heads, self.kv_heads, self.dim
        qkv = self.qkv(x).view(x.shape[0], h + 2 * g, d)
        return qkv[:, :h], qkv[:, h:h + g], qkv[:, h + g:]

    def prompt(self, x, q_start, new):
        """x [tokens, hidden] of all sequences one after another, `new` tokens each (host numbers); returns [tokens, hidden]."""
        starts = torch.tensor(q_start, dtype=torch.int32, device=x.device)
        counts = starts[1:] - starts[:-1]
        own = torch.repeat_interleave(torch.arange(self.seqs, device=x.device), counts.long(), output_size=x.shape[0])
        at = self.positions[own] + torch.arange(x.shape[0], dtype=torch.int32, device=x.device) - starts[own]
        self.lens += counts
        self.positions += counts
        self.longest += max(new)
        q, k, v = self._split(x)
        cache = self.caches[0]
        tman.tman_rope_append(cache, q, k, v, self.lens, q, rope=self.rope, positions=at.contiguous(), q_start=starts, weights=self.weights)
        y = torch.empty_like(q, memory_format=torch.contiguous_format)
        need = tman.tman_attn_prefill_workspace_bytes(cache, self.attn, x.shape[0], self.longest)
        if need > self.workspace.numel():
            self.workspace = torch.zeros(need, dtype=torch.uint8, device=x.device)
        tman.tman_attn_prefill(cache, self.attn, q, starts, self.lens, y, self.longest, self.workspace)
        self.last = q, y  # what went in and came out of the attention
        return self.out(y.view(x.shape[0], -1))

    def step(self, x):
        """One token of every sequence: x [seqs, hidden]; adds the weights of all positions up."""
        at = self.positions.clone()
        self.lens += 1
        self.positions += 1
        self.longest += 1
        q, k, v = self._split(x)
        cache = self.caches[0]
        tman.tman_rope_append(cache, q, k, v, self.lens, q, rope=self.rope, positions=at, weights=self.weights)
        y = torch.empty_like(q, memory_format=torch.contiguous_format)
        tman.tman_attn_decode(cache, self.attn, q, self.lens, y, self.longest, self.workspace, weights=self.weights)
        self.last = q, y
        return self.out(y.view(self.seqs, -1))

    def make_room(self):
        """Keeps the budget of every sequence in the other set of pages and goes on there."""
        new_lens = torch.empty_like(self.lens)
        tman.tman_kv_evict(self.caches[0], self.weights, self.lens, self.budget, self.recent, self.caches[1].page_table, new_lens, self.kept,
                           self.longest)
        self.caches.reverse()
        self.lens, self.longest = new_lens, min(self.longest, self.budget)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("seqs", 4), ("prompt", 300), ("steps", 40), ("budget", 256), ("recent", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    block = AttentionBlock(seqs=a.seqs, most=a.prompt + a.steps, budget=a.budget, recent=a.recent)
    hidden = block.out.shape.M
    new = [max(1, a.prompt - 37 * b) for b in range(a.seqs)]
    starts = [sum(new[:b]) for b in range(a.seqs + 1)]
    x = torch.randn(starts[-1], hidden, device="cuda").half()
    torch.cuda.synchronize()
    t = time.perf_counter()
    y = block.prompt(x, starts, new)
    torch.cuda.synchronize()
    print(f"prompts of {new} tokens: {1e3 * (time.perf_counter() - t):.2f} ms, output {tuple(y.shape)}")
    x = y[[s - 1 for s in starts[1:]]].contiguous()
    t, evictions = time.perf_counter(), 0
    for _ in range(a.steps):
        if block.longest >= a.budget + 32:
            block.make_room()
            evictions += 1
        y = block.step(x)
        x = (y / y.float().square().mean(-1, keepdim=True).sqrt()).half()
    torch.cuda.synchronize()
    print(f"{a.steps} steps of {a.seqs} sequences: {1e3 * (time.perf_counter() - t) / a.steps:.3f} ms each, {evictions} evictions, "
          f"lengths {block.lens.tolist()} of {block.positions.tolist()} positions")
    assert tman.tman_device_status() == 0 and bool(y.isfinite().all())


if __name__ == "__main__":
    main()
