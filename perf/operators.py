"""Timed cases of the operators around a paged key-value cache: what writes it, what reads it, what makes room in it.

A case is one call as a program that serves a decoder makes it:

  op       what one pass does
  append   ``tman_rope_append``: rotates the queries and keys of new tokens (one axis of positions, or time, height and
           width) and writes keys and values into the pages of the cache
  decode   ``tman_attn_decode``: attention of one new token of each sequence over its cache
  prefill  ``tman_attn_prefill``: attention of prompts, or of a chunk of one, over the cache that holds them already
  evict    ``tman_kv_evict``: keeps the positions with the most accumulated attention weight and moves them to new pages

``type`` float16 or bfloat16; ``heads`` query and ``kv_heads`` key-value heads of ``dim``; pages of ``page`` positions;
``seqs`` sequences of up to ``length`` positions (their lengths differ where ``ragged``), ``tokens`` of them new.  Scores may
be capped (``cap``), lowered with the distance (``slopes``), limited to a ``window`` of positions; ``mask`` says what a
query of a prompt sees: everything up to itself (causal), only its own document (documents), a common prefix besides
(prefix).  Lengths and masks come from the case, tensors and the order of the pages from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DEFAULTS = dict(type="float16", heads=32, kv_heads=8, dim=128, page=64, seqs=1, length=1, tokens=1, ragged=False, cap=0.0,
                 slopes=False, window=0, mask="causal", weights=False, axes=1, rot=0, interleaved=False, keep=0, recent=0)


def _case(op, **more):
    return dict(op=op, **{**_DEFAULTS, **more})


def listed():
    return [
        # eight sequences take a step together: their tokens' queries, keys and values (latency of the call)
        dict(name="append_8_tokens", **_case("append", seqs=8, length=2000, ragged=True)),
        # a long clip as a prompt, positions in time, height and width, all heads with keys of their own, recycled pages
        dict(name="append_5461_video", **_case("append", type="bfloat16", heads=32, kv_heads=32, page=16, length=5461,
                                               tokens=5461, axes=3, weights=True)),
        # one short conversation (latency of the call)
        dict(name="decode_1x777", **_case("decode", page=16, length=777)),
        # a batch of conversations of very different lengths, a 7B decoder with as many key-value as query heads
        dict(name="decode_32x4096_ragged", **_case("decode", heads=32, kv_heads=32, seqs=32, length=4096, ragged=True)),
        # two long documents, grouped heads
        dict(name="decode_2x131072", **_case("decode", type="bfloat16", seqs=2, length=131072, page=128)),
        # a batch whose cache will be thinned out later: the weights of the positions are added up; capped scores, a
        # distance bias
        dict(name="decode_16x4095_weights", **_case("decode", heads=16, kv_heads=2, dim=64, page=32, seqs=16, length=4095,
                                                    ragged=True, cap=30.0, slopes=True, weights=True)),
        # three short prompts of a few tokens each
        dict(name="prefill_3_short", **_case("prefill", heads=24, kv_heads=24, page=16, seqs=3, length=33, tokens=33, ragged=True)),
        # a whole prompt with capped scores
        dict(name="prefill_8192_capped", **_case("prefill", type="bfloat16", length=8192, tokens=8192, cap=50.0)),
        # documents packed behind one another, a distance bias, padding at the end (rows that see nothing)
        dict(name="prefill_7001_documents", **_case("prefill", heads=32, kv_heads=32, length=7001, tokens=7001,
                                                    mask="documents", slopes=True)),
        # the next chunk of a long prompt, a part of it seen by all
        dict(name="prefill_2047_at_16384", **_case("prefill", heads=16, kv_heads=2, dim=64, length=16384, tokens=2047,
                                                   mask="prefix")),
        # four conversations reach their budget
        dict(name="evict_4x2049", **_case("evict", page=16, seqs=4, length=2049, keep=1024, recent=128)),
        # a batch of long documents is cut to a quarter
        dict(name="evict_16x16384", **_case("evict", type="bfloat16", seqs=16, length=16384, ragged=True, keep=4096, recent=512)),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    """One more case of the ranges of the listed ones: up to 64 sequences, up to 131072 positions, at most their largest cost."""
    op = rng.choice(["append", "decode", "decode", "prefill", "prefill", "evict"])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 16, 32])
    heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 5, 7, 8, 16) if g * kv_heads <= 64])
    c = _case(op, type=rng.choice(["float16", "bfloat16"]), heads=heads, kv_heads=kv_heads, dim=rng.choice([64, 128, 128, 256]),
              page=rng.choice([16, 32, 64, 128, 256]), ragged=rng.random() < 0.7)
    row = kv_heads * c["dim"] * 4  # bytes of one position's key and value
    if op == "append":
        c["seqs"] = _log(rng, 1, 64)
        c["tokens"] = 1 if rng.random() < 0.5 else _log(rng, 1, 8192 // c["seqs"])
        c["length"] = c["tokens"] + _log(rng, 1, 4096)
        c["axes"] = rng.choice([1, 1, 2, 3])
        c["rot"] = rng.choice([0, c["dim"] // 2])
        c["interleaved"] = rng.random() < 0.5
        c["weights"] = rng.random() < 0.5
        while c["seqs"] * c["tokens"] * (heads + kv_heads) * c["dim"] > 5461 * 64 * 128:
            c["tokens"] = (c["tokens"] + 1) // 2
    elif op == "decode":
        c["seqs"] = _log(rng, 1, 64)
        c["length"] = _log(rng, 1, 131072)
        while c["seqs"] * c["length"] * row > 2 * 131072 * 8 * 512:
            c["length"] = (c["length"] + 1) // 2
        c["cap"] = rng.choice([0.0, 0.0, 30.0])
        c["slopes"] = rng.random() < 0.3
        c["window"] = rng.choice([0, 0, _log(rng, 1, 4096)])
        c["weights"] = rng.random() < 0.3
    elif op == "prefill":
        c["seqs"] = _log(rng, 1, 8)
        c["tokens"] = _log(rng, 1, 8192)
        c["length"] = c["tokens"] + rng.choice([0, 0, _log(rng, 1, 16384)])
        while c["seqs"] * heads * c["dim"] * c["tokens"] * c["length"] > 32 * 128 * 8192 * 8192:
            if c["tokens"] == c["length"]:
                c["tokens"] = c["length"] = (c["tokens"] + 1) // 2
            else:
                c["tokens"] = (c["tokens"] + 1) // 2
                c["length"] = max(c["tokens"], (c["length"] * 3 + 3) // 4)
        c["cap"] = rng.choice([0.0, 0.0, 50.0])
        c["slopes"] = rng.random() < 0.3
        c["window"] = rng.choice([0, 0, _log(rng, 1, 4096)])
        c["mask"] = rng.choice(["causal", "documents", "prefix"])
    else:
        c["seqs"] = _log(rng, 1, 32)
        c["length"] = _log(rng, 32, 65536)
        while c["seqs"] * c["length"] * row > 16 * 16384 * 8 * 512:
            c["length"] = (c["length"] + 1) // 2
        c["keep"] = max(1, int(c["length"] * rng.uniform(0.1, 0.9)))
        c["recent"] = int(c["keep"] * rng.uniform(0.0, 1.0))
    return c


# ---- what the case alone decides: lengths and masks

def _numbers(case):
    return random.Random(case["seqs"] * 1000003 + case["length"] * 101 + case["tokens"])


def _lengths(case):
    """(new tokens, positions with them) of every sequence; the first has the full length."""
    r, new, total = _numbers(case), [], []
    for b in range(case["seqs"]):
        t, n = case["tokens"], case["length"]
        if case["ragged"] and b:
            if case["tokens"] > 1:
                t = r.randint(1, t)
                n = t + r.randint(0, case["length"] - case["tokens"])
            else:
                n = r.randint(1, n)
        new.append(t)
        total.append(n)
    return new, total


def _visible(case):
    """Per new token of a prompt the interval [first, end) of the positions that its mask leaves (without the window)."""
    r = _numbers(case)
    new, total = _lengths(case)
    first, end = [], []
    for t, n in zip(new, total):
        if case["mask"] == "documents":
            starts = sorted({0, *(r.randrange(n) for _ in range(n // 1000 + 1))})
            padding = min(t // 8, 5)  # the last tokens fill the batch up and see nothing
            k = 0
            for i in range(n - t, n):
                while k + 1 < len(starts) and starts[k + 1] <= i:
                    k += 1
                first.append(starts[k] if i < n - padding else n)
                end.append(i + 1)
        else:
            prefix = n * 3 // 4 if case["mask"] == "prefix" else 0
            first += [0] * t
            end += [max(i + 1, prefix) for i in range(n - t, n)]
    return first, end


def _sections(case):
    """Pairs of a head's coordinates that turn with each axis of positions."""
    pairs = (case["rot"] or case["dim"]) // 2
    if case["axes"] == 1:
        return [pairs]
    rest = pairs * 3 // 8
    return [pairs - rest, rest] if case["axes"] == 2 else [pairs - 2 * rest, rest, rest]


def work(case):
    new, total = _lengths(case)
    D, H, G = case["dim"], case["heads"], case["kv_heads"]
    N, S = sum(new), sum(total)
    if case["op"] == "append":
        angles = N * (case["rot"] or D) * 4
        return {"bytes": 2 * N * (H + 2 * G) * D * 2 + angles, "flops": 3 * N * (H + G) * (case["rot"] or D)}
    if case["op"] == "evict":
        kept = sum(min(n, case["keep"]) for n in total)
        return {"bytes": 4 * S * G + 2 * kept * G * (4 * D + 4), "flops": 0}
    if case["op"] == "decode":
        if case["window"]:
            S = sum(min(n, case["window"]) for n in total)
        return {"bytes": S * G * D * 4 + 2 * N * H * D * 2 + 4 * N * H + (8 * S * G if case["weights"] else 0),
                "flops": 4 * S * H * D}
    first, end = _visible(case)
    pairs, seen, t0 = 0, 0, 0
    for t, n in zip(new, total):
        low, high = n, 0
        for i in range(t):
            a, e, at = first[t0 + i], end[t0 + i], n - t + i
            if case["window"]:
                a = max(a, at - case["window"] + 1)
            if a < e:
                pairs += e - a
                low, high = min(low, a), max(high, e)
        seen += max(0, high - low)
        t0 += t
    return {"bytes": seen * G * D * 4 + 2 * N * H * D * 2 + 4 * N * H, "flops": 4 * pairs * H * D}


# ---- inputs

def prepare(case, seed):
    device = torch.device("cuda")
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    dtype = getattr(torch, case["type"])
    D, H, G, P = case["dim"], case["heads"], case["kv_heads"], case["page"]
    new, total = _lengths(case)
    B, N = len(new), sum(new)
    longest = max(total)

    def normal(*shape, dtype=dtype):
        return torch.randn(*shape, generator=gen, device=device, dtype=torch.float32).to(dtype)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=device)

    # pages of all sequences in an arbitrary order, as a cache that has been in use for a while holds them
    wide = (longest + P - 1) // P
    kept_wide = (case["keep"] + P - 1) // P
    n_pages = sum((n + P - 1) // P for n in total) + (B * kept_wide if case["op"] == "evict" else 0) + 3
    order = torch.randperm(n_pages, generator=gen, device=device).to(torch.int32).tolist()
    table, new_table = [], []
    for n in total:
        used = (n + P - 1) // P
        table.append([order.pop() for _ in range(used)] + [0] * (wide - used))
        new_table.append([order.pop() for _ in range(kept_wide)] if case["op"] == "evict" else [])
    s = dict(case=case, new=new, longest=longest, table=ints(table), lens=ints(total),
             k_pages=torch.empty(n_pages, G, P, D, dtype=dtype, device=device),
             v_pages=torch.empty(n_pages, G, P, D, dtype=dtype, device=device), scale=D ** -0.5)
    for pages in (s["k_pages"], s["v_pages"]):
        for at in range(0, n_pages, 1024):
            pages[at:at + 1024] = normal(*pages[at:at + 1024].shape)
    if case["op"] != "evict":
        starts = [0]
        for t in new:
            starts.append(starts[-1] + t)
        s["q_start"] = ints(starts)
        # queries, keys and values as the columns of one fused projection
        qkv = normal(N, H + 2 * G, D)
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
        s["out"] = torch.empty(N, H, D, dtype=dtype, device=device)
        s["lse"] = torch.empty(N, H, dtype=torch.float32, device=device)
    s["slopes"] = None
    if case["slopes"]:
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], dtype=torch.float32, device=device)
    if case["op"] == "evict" or case["weights"]:
        # few positions hold most of the weight; some have none at all (ties)
        w = torch.rand(n_pages, G, P, generator=gen, device=device)
        s["weights"] = torch.where(w < 0.1, torch.zeros_like(w), torch.exp(8 * w) / 100)
    if case["op"] == "append":
        rot = case["rot"] or D
        pos = torch.arange(longest, dtype=torch.float64, device=device)
        freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
        angle = pos[:, None] * freq[None, :]
        s["cos_sin"] = torch.stack([angle.cos(), angle.sin()], dim=-1).to(torch.float32).contiguous()
        s["positions"] = None
        if case["axes"] > 1:
            at = torch.cat([torch.arange(n - t, n, device=device) for t, n in zip(new, total)])
            grid = [at // 256, at % 256 // 16, at % 16]  # frames of 16 x 16 patches
            s["positions"] = torch.stack(grid[:case["axes"]]).to(torch.int32).contiguous()
    if case["op"] == "prefill":
        first, end = _visible(case)
        s["first"] = ints(first) if case["mask"] == "documents" else None
        s["end"] = ints(end) if case["mask"] == "prefix" else None
    if case["op"] == "evict":
        s["new_table"] = ints(new_table)
        s["new_lens"] = torch.empty(B, dtype=torch.int32, device=device)
        s["kept"] = torch.empty(B, G, case["keep"], dtype=torch.int32, device=device)
    if own:  # the handles and the workspace that a program keeps from call to call
        import paper_2511_11248_amd as tman

        s["cache"] = tman.KvCache(s["k_pages"], s["v_pages"], s["table"])
        if case["op"] == "append":
            s["rope"] = tman.Rope(s["cos_sin"], _sections(case), case["interleaved"])
        if case["op"] in ("decode", "prefill"):
            s["attn"] = tman.Attn(H, s["scale"], cap=case["cap"], window=case["window"], slopes=s["slopes"])
        if case["op"] == "decode":
            need = tman.tman_attn_decode_workspace_bytes(s["cache"], s["attn"], longest, case["weights"])
            s["workspace"] = torch.zeros(need, dtype=torch.uint8, device=device)
        if case["op"] == "prefill":
            need = tman.tman_attn_prefill_workspace_bytes(s["cache"], s["attn"], N, longest)
            s["workspace"] = torch.zeros(need, dtype=torch.uint8, device=device) if need else None
    return s


def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    return {"append": _append, "decode": _decode, "prefill": _prefill, "evict": _evict}[case["op"]](state, case)


def _run_own(s, case):
    import paper_2511_11248_amd as tman

    if case["op"] == "append":
        tman.tman_rope_append(s["cache"], s["q"], s["k"], s["v"], s["lens"], s["out"], rope=s["rope"], positions=s["positions"],
                              q_start=s["q_start"], weights=s.get("weights"))
        return _append_outputs(s, s["out"])
    if case["op"] == "decode":
        tman.tman_attn_decode(s["cache"], s["attn"], s["q"], s["lens"], s["out"], s["longest"], s["workspace"], lse=s["lse"],
                              weights=s.get("weights"))
        return [s["out"], s["lse"]] + ([s["weights"]] if case["weights"] else [])
    if case["op"] == "prefill":
        tman.tman_attn_prefill(s["cache"], s["attn"], s["q"], s["q_start"], s["lens"], s["out"], s["longest"], s["workspace"],
                               first=s["first"], end=s["end"], lse=s["lse"])
        return [s["out"], s["lse"]]
    tman.tman_kv_evict(s["cache"], s["weights"], s["lens"], case["keep"], case["recent"], s["new_table"], s["new_lens"], s["kept"],
                       s["longest"])
    return [s["kept"], s["new_lens"], s["k_pages"], s["v_pages"], s["weights"]]


def _append_outputs(s, q):
    return [q, s["k_pages"], s["v_pages"]] + ([s["weights"]] if s["case"]["weights"] else [])


# ---- plain forms

def _owners(s):
    """Sequence and position of every new token, [N] each."""
    counts = s["q_start"][1:] - s["q_start"][:-1]
    N = s["q"].shape[0]
    b = torch.repeat_interleave(torch.arange(counts.numel(), device=counts.device), counts.long(), output_size=N)
    i = torch.arange(N, device=counts.device) - s["q_start"][b].long()
    return b, s["lens"][b].long() - counts[b].long() + i, i


def _rotate(x, cos, sin, rot, interleaved):
    """x [N, heads, dim] in 32 bits; cos, sin [N, 1, rot / 2]."""
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, a * sin + b * cos
    return y


def _append(s, case):
    dtype, P = s["k_pages"].dtype, case["page"]
    rot = case["rot"] or case["dim"]
    b, at, _ = _owners(s)
    positions = at[None] if s["positions"] is None else s["positions"].long()
    pairs = torch.arange(rot // 2, device=at.device)
    axis = torch.bucketize(pairs, torch.tensor(_sections(case)).cumsum(0).to(at.device), right=True)
    cs = s["cos_sin"][positions[axis].t(), pairs]  # [N, rot / 2, 2]
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    q = _rotate(s["q"].float(), cos, sin, rot, case["interleaved"]).to(dtype)
    k = _rotate(s["k"].float(), cos, sin, rot, case["interleaved"]).to(dtype)
    page, slot = s["table"][b, at // P].long(), at % P
    s["k_pages"][page, :, slot] = k
    s["v_pages"][page, :, slot] = s["v"]
    if case["weights"]:
        s["weights"][page, :, slot] = 0.0
    return _append_outputs(s, q)


def _rows(pages, table):
    """Pages [n_pages, heads, page, ...] of table [B, wide] as rows [B, heads, wide * page, ...]."""
    x = pages[table.long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, *x.shape[4:])


def _softmax_sums(scores, visible, v):
    """sum of softmax(scores) v over the visible positions, their weights and log-sum-exp; a row that sees nothing gives zeros."""
    scores = scores.masked_fill_(~visible, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1)
    p = p.div_(torch.where(total > 0, total, torch.ones_like(total)))
    return p @ v, p, lse


def _bent(s, case, scores, distance):
    """Cap and distance bias on scores [..., heads in a group, ...]; `distance` and the slopes broadcast to them."""
    scores = scores.mul_(s["scale"])
    if case["cap"]:
        scores = scores.div_(case["cap"]).tanh_().mul_(case["cap"])
    if s["slopes"] is not None:
        slopes = s["slopes"].view(1, case["kv_heads"], -1, 1, 1)
        scores = scores.sub_(slopes * distance)
    return scores


def _decode(s, case):
    D, H, G, P = case["dim"], case["heads"], case["kv_heads"], case["page"]
    k, v = _rows(s["k_pages"], s["table"]).float(), _rows(s["v_pages"], s["table"]).float()
    B, S = k.shape[0], k.shape[2]
    j = torch.arange(S, device=k.device)
    n = s["lens"].long()[:, None]
    visible = j < n
    if case["window"]:
        visible = visible & (j > n - 1 - case["window"])
    q = s["q"].float().reshape(B, G, H // G, D)
    scores = (q @ k.transpose(2, 3)).unsqueeze(3)  # [B, G, heads in a group, 1, S]
    scores = _bent(s, case, scores, (n - 1 - j).abs().view(B, 1, 1, 1, S)).squeeze(3)
    v = torch.where(visible.view(B, 1, S, 1), v, torch.zeros_like(v))
    out, p, lse = _softmax_sums(scores, visible.view(B, 1, 1, S), v)
    found = [out.reshape(B, H, D).to(s["q"].dtype), lse.reshape(B, H)]
    if case["weights"]:
        page, slot = s["table"][:, j // P].long(), (j % P).expand(B, S)
        add = p.sum(2).transpose(1, 2)[visible]
        at = (page[visible], slice(None), slot[visible])
        s["weights"][at] = s["weights"][at] + add
        found.append(s["weights"])
    return found


def _prefill(s, case):
    D, H, G = case["dim"], case["heads"], case["kv_heads"]
    k, v = _rows(s["k_pages"], s["table"]).float(), _rows(s["v_pages"], s["table"]).float()
    B, S, T = k.shape[0], k.shape[2], max(s["new"])
    b, at, i = _owners(s)
    j = torch.arange(S, device=k.device)
    n = s["lens"].long()
    end = at + 1 if s["end"] is None else s["end"].long()
    first = torch.zeros_like(at) if s["first"] is None else s["first"].long()
    if case["window"]:
        first = torch.maximum(first, at + 1 - case["window"])
    end = torch.minimum(end, n[b])
    q = torch.zeros(B, T, H, D, device=k.device)
    q[b, i] = s["q"].float()
    q = q.view(B, T, G, H // G, D).permute(0, 2, 3, 1, 4).reshape(B, G, H // G * T, D)
    visible = torch.zeros(B, T, S, dtype=torch.bool, device=k.device)
    visible[b, i] = (j >= first[:, None]) & (j < end[:, None])
    where = torch.zeros(B, T, dtype=torch.long, device=k.device)
    where[b, i] = at
    scores = (q @ k.transpose(2, 3)).view(B, G, H // G, T, S)
    scores = _bent(s, case, scores, (where[:, :, None] - j).abs().view(B, 1, 1, T, S) if case["slopes"] else None)
    v = torch.where((j < n[:, None]).view(B, 1, S, 1), v, torch.zeros_like(v))
    out, _, lse = _softmax_sums(scores, visible.view(B, 1, 1, T, S), v.unsqueeze(2))
    out = out.permute(0, 3, 1, 2, 4).reshape(B, T, H, D)[b, i]
    return [out.to(s["q"].dtype), lse.permute(0, 3, 1, 2).reshape(B, T, H)[b, i]]


def _evict(s, case):
    P, keep, recent = case["page"], case["keep"], case["recent"]
    w = _rows(s["weights"], s["table"])  # [B, G, S]
    B, G, S = w.shape
    j = torch.arange(S, device=w.device)
    n = s["lens"].long().view(B, 1, 1)
    key = torch.where(j < n - recent, w, torch.full_like(w, math.inf))
    key = torch.where(j < n, key, torch.full_like(w, -math.inf))
    if S < keep:
        key = torch.cat([key, torch.full((B, G, keep - S), -math.inf, device=w.device)], dim=2)
    chosen = key.sort(dim=2, descending=True, stable=True).indices[:, :, :keep].sort(dim=2).values
    chosen = torch.where(chosen < n, chosen, torch.full_like(chosen, -1))
    s["kept"].copy_(chosen)
    new_n = s["lens"].clamp(max=keep)
    s["new_lens"].copy_(new_n)
    b, r = torch.nonzero(torch.arange(keep, device=w.device) < new_n[:, None], as_tuple=True)
    g = torch.arange(G, device=w.device)
    src = chosen.transpose(1, 2)[b, r]  # [rows, G]
    src_page, dst_page = s["table"][b[:, None], src // P].long(), s["new_table"][b, r // P].long()
    for_all = (dst_page[:, None], g[None], (r % P)[:, None])
    s["k_pages"][for_all] = s["k_pages"][src_page, g[None], src % P]
    s["v_pages"][for_all] = s["v_pages"][src_page, g[None], src % P]
    s["weights"][for_all] = s["weights"][src_page, g[None], src % P]
    return [s["kept"], s["new_lens"], s["k_pages"], s["v_pages"], s["weights"]]


# ---- the definition in 64 bits, one sequence at a time

def exact(case, seed):
    s = prepare(case, seed)
    D, H, G, P = case["dim"], case["heads"], case["kv_heads"], case["page"]
    R = H // G
    new, total = _lengths(case)
    starts = [sum(new[:b]) for b in range(len(new))]
    if case["op"] == "evict":
        return None  # copies and whole numbers: nothing is computed

    def rows(pages, b, n):  # [G, n, D]
        used = s["table"][b, :(n + P - 1) // P].long()
        return torch.cat(list(pages[used].double()), dim=1)[:, :n]

    if case["op"] == "append":
        rot, out = case["rot"] or D, []
        for b, (t, n) in enumerate(zip(new, total)):
            at = torch.arange(n - t, n, device=s["q"].device)
            tokens = slice(starts[b], starts[b] + t)
            axes = [at] if s["positions"] is None else [a[tokens].long() for a in s["positions"]]
            c, e, p0 = [], [], 0
            for a, count in zip(axes, _sections(case)):
                c.append(s["cos_sin"][a, p0:p0 + count, 0].double())
                e.append(s["cos_sin"][a, p0:p0 + count, 1].double())
                p0 += count
            turn = torch.complex(torch.cat(c, 1), torch.cat(e, 1))[:, None]

            def turned(x):
                x = x.double()
                if case["interleaved"]:
                    z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2).contiguous()) * turn
                    return torch.cat([torch.view_as_real(z).reshape(*x.shape[:-1], rot), x[..., rot:]], -1)
                z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
                return torch.cat([z.real, z.imag, x[..., rot:]], -1)

            out.append(turned(s["q"][tokens]))
            if b == 0:
                k_pages = s["k_pages"].double()
            k_new = turned(s["k"][tokens])
            used = s["table"][b].long()[at // P]
            k_pages[used, :, at % P] = k_new
        return [torch.cat(out), k_pages, None] + ([None] if case["weights"] else [])

    outs, lses = [], []
    total_weights = s["weights"].double() if case["weights"] else None
    slopes = None if s["slopes"] is None else s["slopes"].double()
    if case["op"] == "decode":
        first, end = [0] * len(total), list(total)
    else:
        first, end = _visible(case)
    for b, (t, n) in enumerate(zip(new, total)):
        k, v = rows(s["k_pages"], b, n), rows(s["v_pages"], b, n)
        tokens = slice(starts[b], starts[b] + t)
        lo = torch.tensor(first[tokens], device=k.device)[:, None]
        hi = torch.tensor(end[tokens], device=k.device)[:, None]
        at = torch.arange(n - t, n, device=k.device)[:, None]
        j = torch.arange(n, device=k.device)[None]
        hidden = (j < lo) | (j >= hi)
        if case["window"]:
            hidden = hidden | (j <= at - case["window"])
        out = torch.zeros(t, H, D, dtype=torch.float64, device=k.device)
        lse = torch.zeros(t, H, dtype=torch.float64, device=k.device)
        for h in range(H):
            x = s["q"][tokens, h].double() @ k[h // R].t().contiguous() * s["scale"]
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            if slopes is not None:
                x = x - slopes[h] * (at - j).abs()
            x = x.masked_fill(hidden, -math.inf)
            lse[:, h] = torch.logsumexp(x, 1)
            p = torch.exp(x - lse[:, h:h + 1]).nan_to_num(0.0)  # a row that sees nothing: zeros
            out[:, h] = p @ v[h // R]
            if total_weights is not None:
                total_weights[s["table"][b].long()[j[0] // P], h // R, j[0] % P] += p[0]
        outs.append(out)
        lses.append(lse)
    found = [torch.cat(outs), torch.cat(lses)]
    return found + ([total_weights] if total_weights is not None else [])
