"""Timed cases of what serves a decoder with an 8-bit key-value cache: the pages that a step needs, the append with norms of
queries and keys, and the append to and attention over a cache held in 8 bits.

A case is one call as a program that serves a decoder makes it:

  op       what one pass does
  plan     ``tman_kv_plan``: gives pages to the sequences that grow, takes those of the ones that shrink or end, and says
           where every new token lies (page table, slots, positions, owners)
  norm     ``tman_norm_rope_append``: root-mean-square norm of each query and key head, rotation, append to a 16-bit cache
  append8  ``tman_kv8_append``: the same into a cache of e4m3 codes, with one power of two for each block of 16 positions and head
  decode8  ``tman_attn_decode_kv8``: attention of one new token of each sequence over such a cache
  prefill8 ``tman_attn_prefill_kv8``: attention of prompts, or of a chunk of one, over such a cache

``type`` float16 or bfloat16 (of queries, outputs and new tokens); ``heads`` query and ``kv_heads`` key-value heads of ``dim``;
pages of ``page`` positions; ``seqs`` sequences of up to ``length`` positions (their lengths differ where ``ragged``), ``tokens``
of them new.  ``normed``: heads are normed; ``per_head``: with weights of their own.  Scores may be capped (``cap``), lowered with
the distance (``slopes``), limited to a ``window`` of positions; ``mask`` says what a query of a prompt sees: everything up to
itself (causal), only its own document (documents), a common prefix besides (prefix).  ``scarce``: there are too few free pages
for all.  Lengths and masks come from the case, tensors and the order of the pages from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 16  # positions that share a power of two
_DEFAULTS = dict(type="float16", heads=32, kv_heads=8, dim=128, page=64, seqs=1, length=1, tokens=1, ragged=False, cap=0.0,
                 slopes=False, window=0, mask="causal", axes=1, rot=0, interleaved=False, normed=False, per_head=False,
                 scarce=False)
_EPS = 1e-6


def _case(op, **more):
    return dict(op=op, **{**_DEFAULTS, **more})


def listed():
    return [
        # a decode step of eight sequences: a token each, some need a page (latency of the call)
        dict(name="plan_8_tokens", **_case("plan", seqs=8, length=2000, ragged=True)),
        # a server's queue: prompts and chunks of very different lengths come in, others end, and pages run out
        dict(name="plan_1000_sequences", **_case("plan", seqs=1000, length=4099, tokens=1024, page=16, ragged=True, scarce=True)),
        # eight sequences take a step together, heads normed with one set of weights (latency of the call)
        dict(name="norm_8_tokens", **_case("norm", seqs=8, length=2000, ragged=True, normed=True)),
        # a long prompt, grouped heads
        dict(name="norm_4099", **_case("norm", type="bfloat16", length=4099, tokens=4099, page=128, normed=True, rot=64)),
        # eight sequences take a step together: their blocks hold older positions (latency of the call)
        dict(name="append8_8_tokens", **_case("append8", seqs=8, length=2000, ragged=True)),
        # three long clips as prompts, positions in time, height and width, normed heads with keys of their own
        dict(name="append8_3x2731_video", **_case("append8", type="bfloat16", heads=32, kv_heads=32, page=16, seqs=3, length=2731,
                                                  tokens=2731, axes=3, normed=True, per_head=True)),
        # one short conversation (latency of the call)
        dict(name="decode8_1x777", **_case("decode8", page=16, length=777)),
        # a batch of conversations of very different lengths, a 7B decoder with as many key-value as query heads
        dict(name="decode8_32x4096_ragged", **_case("decode8", heads=32, kv_heads=32, seqs=32, length=4096, ragged=True)),
        # two long documents, grouped heads
        dict(name="decode8_2x131072", **_case("decode8", type="bfloat16", seqs=2, length=131072, page=128)),
        # a few proposed tokens are checked against a long cache, capped scores
        dict(name="prefill8_5_at_16384", **_case("prefill8", seqs=2, length=16384, tokens=5, cap=30.0)),
        # a whole prompt
        dict(name="prefill8_8192", **_case("prefill8", type="bfloat16", length=8192, tokens=8192)),
        # the next chunk of a long prompt, a distance bias, a part of it seen by all
        dict(name="prefill8_2047_at_16384", **_case("prefill8", heads=16, kv_heads=2, length=16384, tokens=2047, mask="prefix",
                                                    slopes=True)),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    """One more case of the ranges of the listed ones: up to 64 sequences (2000 where pages are given), up to 131072 positions, at
    most their largest cost."""
    op = rng.choice(["plan", "norm", "append8", "append8", "decode8", "decode8", "prefill8", "prefill8"])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 16, 32])
    heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 5, 7, 8, 16) if g * kv_heads <= 64])
    c = _case(op, type=rng.choice(["float16", "bfloat16"]), heads=heads, kv_heads=kv_heads, dim=rng.choice([64, 128, 128, 256]),
              page=rng.choice([16, 32, 64, 128, 256]), ragged=rng.random() < 0.7)
    row = kv_heads * c["dim"] * 2  # bytes of one position's key and value
    if op == "plan":
        c["seqs"] = _log(rng, 1, 2000)
        c["tokens"] = 1 if rng.random() < 0.4 else _log(rng, 1, max(1, 400000 // c["seqs"]))
        c["length"] = c["tokens"] + _log(rng, 1, 8192)
        c["ragged"] = True
        c["scarce"] = rng.random() < 0.3
    elif op in ("norm", "append8"):
        c["seqs"] = _log(rng, 1, 64)
        c["tokens"] = 1 if rng.random() < 0.4 else _log(rng, 1, 8192 // c["seqs"])
        c["length"] = c["tokens"] + _log(rng, 1, 4096)
        c["axes"] = rng.choice([1, 1, 2, 3])
        c["rot"] = rng.choice([0, c["dim"] // 2])
        c["interleaved"] = rng.random() < 0.5
        c["normed"] = op == "norm" or rng.random() < 0.5
        c["per_head"] = c["normed"] and rng.random() < 0.3
        while c["seqs"] * c["tokens"] * (heads + kv_heads) * c["dim"] > 4099 * 40 * 128:
            c["tokens"] = (c["tokens"] + 1) // 2
    elif op == "decode8":
        c["seqs"] = _log(rng, 1, 64)
        c["length"] = _log(rng, 1, 131072)
        while c["seqs"] * c["length"] * row > 2 * 131072 * 8 * 256:
            c["length"] = (c["length"] + 1) // 2
        c["cap"] = rng.choice([0.0, 0.0, 30.0])
        c["slopes"] = rng.random() < 0.3
        c["window"] = rng.choice([0, 0, _log(rng, 1, 4096)])
    else:
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


def _changes(case):
    """A plan's (positions before, tokens that come or, below zero, positions that go) of every sequence: a sixth of them end or
    lose their last positions, a few do nothing."""
    r = _numbers(case)
    new, total = _lengths(case)
    before, more = [], []
    for b, (t, n) in enumerate(zip(new, total)):
        held = n - t
        kind = r.random() if b else 1.0
        before.append(held)
        more.append(-held if kind < 0.12 else -min(held, r.randint(1, 8)) if kind < 0.17 else 0 if kind < 0.2 else t)
    return before, more


def _free_pages(case):
    """Pages that are free before a plan: a little more than it takes, or about half of that."""
    P = case["page"]
    before, more = _changes(case)
    need = sum(max(0, -(-(n + m) // P) + (-n // P)) for n, m in zip(before, more))
    back = sum(max(0, -(-n // P) + (-(n + m) // P)) for n, m in zip(before, more))
    return max(0, need // 2 - back) if case["scarce"] else need + 5


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
    D, H, G, P = case["dim"], case["heads"], case["kv_heads"], case["page"]
    if case["op"] == "plan":
        before, more = _changes(case)
        N = sum(max(0, m) for m in more)
        pages = sum(abs(-(-(n + m) // P) + (-n // P)) for n, m in zip(before, more))
        return {"bytes": 16 * len(more) + 8 * pages + 16 * N, "flops": 0}
    new, total = _lengths(case)
    N, S = sum(new), sum(total)
    if case["op"] in ("norm", "append8"):
        held = 2 if case["op"] == "norm" else 1
        rot = case["rot"] or D
        return {"bytes": N * D * (4 * H + 2 * G * (2 + held)) + N * rot * 4, "flops": N * (H + G) * (3 * rot + (4 * D if case["normed"] else 0))}
    if case["op"] == "decode8":
        if case["window"]:
            S = sum(min(n, case["window"]) for n in total)
        return {"bytes": S * G * D * 2 + S * G // 8 + 2 * N * H * D * 2 + 4 * N * H, "flops": 4 * S * H * D}
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
    return {"bytes": seen * G * D * 2 + seen * G // 8 + 2 * N * H * D * 2 + 4 * N * H, "flops": 4 * pairs * H * D}


# ---- inputs

def prepare(case, seed):
    device = torch.device("cuda")
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    dtype = getattr(torch, case["type"])
    D, H, G, P = case["dim"], case["heads"], case["kv_heads"], case["page"]
    B = case["seqs"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=device, dtype=torch.float32)

    def ints(values, dtype=torch.int32):
        return torch.tensor(values, dtype=dtype, device=device)

    if case["op"] == "plan":
        before, more = _changes(case)
        used = [-(-n // P) for n in before]
        free = _free_pages(case)
        wide = max(-(-max(n, n + m) // P) for n, m in zip(before, more)) + 1
        order = torch.randperm(sum(used) + free, generator=gen, device=device).to(torch.int32).tolist()
        table = [[order.pop() for _ in range(u)] + [0] * (wide - u) for u in used]
        N = max(1, sum(max(0, m) for m in more))
        N += N // 16  # a padded batch
        s = dict(case=case, table=ints(table), lens=ints(before), more=ints(more), free_left=ints([free]),
                 free_pages=ints(order + [-1] * sum(used)), new_lens=torch.empty(B, dtype=torch.int32, device=device),
                 new_left=torch.empty(1, dtype=torch.int32, device=device), q_start=torch.empty(B + 1, dtype=torch.int32, device=device),
                 slots=torch.empty(N, dtype=torch.int64, device=device), positions=torch.empty(N, dtype=torch.int32, device=device),
                 owners=torch.empty(N, dtype=torch.int32, device=device))
        if own:  # the workspace that a program keeps from call to call
            import paper_2511_11248_amd as tman

            s["workspace"] = torch.empty(max(1, tman.tman_kv_plan_workspace_bytes(B, N)), dtype=torch.uint8, device=device)
        return s

    new, total = _lengths(case)
    N, longest = sum(new), max(total)
    # pages of all sequences in an arbitrary order, as a cache that has been in use for a while holds them
    wide = (longest + P - 1) // P
    n_pages = sum((n + P - 1) // P for n in total) + 3
    order = torch.randperm(n_pages, generator=gen, device=device).to(torch.int32).tolist()
    table = []
    for n in total:
        held = (n + P - 1) // P
        table.append([order.pop() for _ in range(held)] + [0] * (wide - held))
    held8 = case["op"] != "norm"
    kind = torch.float8_e4m3fn if held8 else dtype
    s = dict(case=case, new=new, longest=longest, table=ints(table), lens=ints(total), scale=D ** -0.5,
             k_pages=torch.empty(n_pages, G, P, D, dtype=kind, device=device),
             v_pages=torch.empty(n_pages, G, P, D, dtype=kind, device=device))
    for pages in (s["k_pages"], s["v_pages"]):
        for at in range(0, n_pages, 1024):
            x = normal(*pages[at:at + 1024].shape)
            pages[at:at + 1024] = (x * 90).clamp_(-448, 448).to(kind) if held8 else x.to(kind)
    if held8:  # values of about one, some blocks with larger or smaller ones
        for name in ("k_exps", "v_exps"):
            s[name] = torch.randint(119, 123, (n_pages, G, P // BLOCK), generator=gen, device=device, dtype=torch.uint8)
    starts = [0]
    for t in new:
        starts.append(starts[-1] + t)
    s["q_start"] = ints(starts)
    # queries, keys and values as the columns of one fused projection
    qkv = normal(N, H + 2 * G, D)
    if case["op"] in ("norm", "append8"):
        qkv *= torch.exp(0.7 * normal(N, 1, 1))  # tokens differ in size
    qkv = qkv.to(dtype)
    s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
    s["out"] = torch.empty(N, H, D, dtype=dtype, device=device)
    s["lse"] = torch.empty(N, H, dtype=torch.float32, device=device)
    s["slopes"] = None
    if case["slopes"]:
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], dtype=torch.float32, device=device)
    if case["op"] in ("norm", "append8"):
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
        if case["normed"]:
            s["q_weight"] = 1 + 0.3 * normal(*((H, D) if case["per_head"] else (D,)))
            s["k_weight"] = 1 + 0.3 * normal(*((G, D) if case["per_head"] else (D,)))
    if case["op"] == "prefill8":
        first, end = _visible(case)
        s["first"] = ints(first) if case["mask"] == "documents" else None
        s["end"] = ints(end) if case["mask"] == "prefix" else None
    if own:  # the handles and the workspace that a program keeps from call to call
        import paper_2511_11248_amd as tman

        if held8:
            s["cache"] = tman.KvCache8(s["k_pages"], s["v_pages"], s["k_exps"], s["v_exps"], s["table"], dtype)
        else:
            s["cache"] = tman.KvCache(s["k_pages"], s["v_pages"], s["table"])
        if case["op"] in ("norm", "append8"):
            s["rope"] = tman.Rope(s["cos_sin"], _sections(case), case["interleaved"])
            s["norm"] = tman.HeadNorm(s["q_weight"], s["k_weight"], _EPS) if case["normed"] else None
        else:
            s["attn"] = tman.Attn(H, s["scale"], cap=case["cap"], window=case["window"], slopes=s["slopes"])
            if case["op"] == "decode8":
                need = tman.tman_attn_decode_kv8_workspace_bytes(s["cache"], s["attn"], longest)
            else:
                need = tman.tman_attn_prefill_kv8_workspace_bytes(s["cache"], s["attn"], N, longest)
            s["workspace"] = torch.zeros(need, dtype=torch.uint8, device=device) if need else None
    return s


def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    return {"plan": _plan, "norm": _norm, "append8": _append8, "decode8": _decode8, "prefill8": _prefill8}[case["op"]](state, case)


def _run_own(s, case):
    import paper_2511_11248_amd as tman

    if case["op"] == "plan":
        tman.tman_kv_plan(s["table"], case["page"], s["lens"], s["more"], s["free_pages"], s["free_left"], s["new_lens"], s["new_left"],
                          s["q_start"], s["slots"], s["positions"], s["owners"], s["workspace"])
        return _plan_outputs(s)
    if case["op"] == "norm":
        tman.tman_norm_rope_append(s["cache"], s["norm"], s["q"], s["k"], s["v"], s["lens"], s["out"], rope=s["rope"],
                                   positions=s["positions"], q_start=s["q_start"])
        return [s["out"], s["k_pages"], s["v_pages"]]
    if case["op"] == "append8":
        tman.tman_kv8_append(s["cache"], s["q"], s["k"], s["v"], s["lens"], s["out"], norm=s["norm"], rope=s["rope"],
                             positions=s["positions"], q_start=s["q_start"])
        return [s["out"], s["k_pages"], s["v_pages"], s["k_exps"], s["v_exps"]]
    if case["op"] == "decode8":
        tman.tman_attn_decode_kv8(s["cache"], s["attn"], s["q"], s["lens"], s["out"], s["longest"], s["workspace"], lse=s["lse"])
        return [s["out"], s["lse"]]
    tman.tman_attn_prefill_kv8(s["cache"], s["attn"], s["q"], s["q_start"], s["lens"], s["out"], s["longest"], s["workspace"],
                               first=s["first"], end=s["end"], lse=s["lse"])
    return [s["out"], s["lse"]]


def _plan_outputs(s):
    return [s[name] for name in ("table", "new_lens", "new_left", "q_start", "slots", "positions", "owners", "free_pages")]


# ---- plain forms

def _plan(s, case):
    P, table, stack = case["page"], s["table"], s["free_pages"]
    lens, more, left = s["lens"].long(), s["more"].long(), s["free_left"].long()
    N, wide = s["slots"].numel(), table.shape[1]
    old = (lens + P - 1) // P
    now = (lens + more + P - 1) // P
    # what is given back goes onto the stack, in order
    entry = torch.arange(wide, device=lens.device)
    back = (entry >= now[:, None]) & (entry < old[:, None])
    given = back.flatten().cumsum(0)
    at = left + given - 1
    # (entries that stay write to a place behind the stack)
    longer = torch.cat([stack, stack.new_zeros(1)])
    longer[torch.where(back.flatten(), at, torch.full_like(at, stack.numel()))] = table.flatten()
    stack.copy_(longer[:-1])
    left = left + given[-1]
    # what is taken comes from its top, in order, as long as it lasts
    need = (now - old).clamp(min=0)
    taken = need.cumsum(0)
    granted = (more > 0) & ((need == 0) | (taken <= left)) & (more.clamp(min=0).cumsum(0) <= N)
    got = torch.where(granted, need, torch.zeros_like(need))
    base = left - 1 - (taken - need)
    k = entry - old[:, None]
    fresh = (k >= 0) & (k < got[:, None])
    table.copy_(torch.where(fresh, stack[(base[:, None] - k).clamp(min=0)], table))
    s["new_left"].copy_(left - got.sum())
    change = torch.where(granted | (more < 0), more, torch.zeros_like(more))
    s["new_lens"].copy_(lens + change)
    starts = torch.cat([left.new_zeros(1), change.clamp(min=0).cumsum(0)])
    s["q_start"].copy_(starts)
    n = torch.arange(N, device=lens.device)
    owner = torch.searchsorted(starts, n, right=True) - 1
    valid = n < starts[-1]
    owner = owner.clamp(max=lens.numel() - 1)
    position = lens[owner] + n - starts[owner]
    page = table[owner, torch.where(valid, position // P, torch.zeros_like(position))].long()
    none = torch.full_like(n, -1)
    s["slots"].copy_(torch.where(valid, page * P + position % P, none))
    s["positions"].copy_(torch.where(valid, position, none))
    s["owners"].copy_(torch.where(valid, owner, none))
    return _plan_outputs(s)


def _owners(s):
    """Sequence and position of every new token, [N] each."""
    counts = s["q_start"][1:] - s["q_start"][:-1]
    N = s["q"].shape[0]
    b = torch.repeat_interleave(torch.arange(counts.numel(), device=counts.device), counts.long(), output_size=N)
    i = torch.arange(N, device=counts.device) - s["q_start"][b].long()
    return b, s["lens"][b].long() - counts[b].long() + i, i


def _rotate(x, cos, sin, rot, interleaved):
    """x [N, heads, dim]; cos, sin [N, 1, rot / 2]."""
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, a * sin + b * cos
    return y


def _normed(x, weight):
    return x * ((x * x).mean(-1, keepdim=True) + _EPS).rsqrt() * weight


def _turned(s, case, at, wide):
    """Normed and rotated queries in 32 bits and keys in type `wide`."""
    rot = case["rot"] or case["dim"]
    positions = at[None] if s["positions"] is None else s["positions"].long()
    pairs = torch.arange(rot // 2, device=at.device)
    axis = torch.bucketize(pairs, torch.tensor(_sections(case)).cumsum(0).to(at.device), right=True)
    cs = s["cos_sin"][positions[axis].t(), pairs]  # [N, rot / 2, 2]
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    q, k = s["q"].float(), s["k"].to(wide)
    if case["normed"]:
        q, k = _normed(q, s["q_weight"]), _normed(k, s["k_weight"].to(wide))
    return (_rotate(q, cos, sin, rot, case["interleaved"]),
            _rotate(k, cos.to(wide), sin.to(wide), rot, case["interleaved"]))


def _norm(s, case):
    P, dtype = case["page"], s["k_pages"].dtype
    b, at, _ = _owners(s)
    q, k = _turned(s, case, at, torch.float32)
    page, slot = s["table"][b, at // P].long(), at % P
    s["k_pages"][page, :, slot] = k.to(dtype)
    s["v_pages"][page, :, slot] = s["v"]
    return [q.to(dtype), s["k_pages"], s["v_pages"]]


def _exponents(largest):
    """The least e with largest <= 448 * 2^e, biased by 127, at least 10 (448 = 7/8 * 2^9)."""
    part, e = torch.frexp(largest)
    e = e.long() - 9 + (part > 0.875)
    return torch.where(largest > 0, e + 127, torch.zeros_like(e)).clamp(min=10)


def _power(e):
    """2^(e - 127), 1 <= e <= 254, out of its bits."""
    return (e.int() << 23).view(torch.float32)


def _codes(x, e):
    """x / 2^(e - 127) as the nearest e4m3 codes, as bytes; x has no infinities here."""
    return (x * _power(254 - e)).clamp(-448, 448).float().to(torch.float8_e4m3fn).view(torch.uint8)


def _append8(s, case):
    P, D, dtype = case["page"], case["dim"], s["q"].dtype
    b, at, _ = _owners(s)
    q, k = _turned(s, case, at, torch.float64)  # (64 bits: the largest value of a block decides over all its codes)
    page, slot = s["table"][b, at // P].long(), at % P
    g = torch.arange(case["kv_heads"], device=at.device)
    # older positions of the sequences' first blocks
    counts = (s["q_start"][1:] - s["q_start"][:-1]).long()
    begin = s["lens"].long() - counts
    block = begin // BLOCK * BLOCK
    row = block[:, None] + torch.arange(BLOCK, device=at.device)
    owner, which = torch.nonzero((row < begin[:, None]) & (counts[:, None] > 0), as_tuple=True)
    row = row[owner, which]
    old_page, old_slot = s["table"][owner, row // P].long(), row % P
    for x, pages, exps in ((k, s["k_pages"], s["k_exps"]), (s["v"].double(), s["v_pages"], s["v_exps"])):
        codes, P16 = pages.view(torch.uint8), P // BLOCK
        place = ((page[:, None] * case["kv_heads"] + g) * P16 + (slot // BLOCK)[:, None]).flatten()
        largest = torch.zeros(exps.numel(), dtype=x.dtype, device=x.device).scatter_reduce_(0, place, x.abs().amax(-1).flatten(), "amax")
        before = exps.long()
        e = torch.zeros(exps.numel(), dtype=torch.long, device=x.device)
        e[place] = _exponents(largest)[place]
        e = e.view_as(before)
        e[old_page, :, old_slot // BLOCK] = torch.maximum(e, before)[old_page, :, old_slot // BLOCK]
        values = codes[old_page, :, old_slot].view(torch.float8_e4m3fn).double()
        shift = 127 + (e - before)[old_page, :, old_slot // BLOCK]
        codes[old_page, :, old_slot] = _codes(values, shift[..., None])
        codes[page, :, slot] = _codes(x, e[page, :, slot // BLOCK][..., None])
        exps.copy_(torch.where(e > 0, e, before))
    return [q.to(dtype), s["k_pages"], s["v_pages"], s["k_exps"], s["v_exps"]]


def _values(pages, exps, table):
    """The values that pages of table [B, wide] hold, as rows [B, heads, wide * page, dim] in 32 bits."""
    table = table.long()
    x = pages.view(torch.uint8)[table].view(torch.float8_e4m3fn).float()
    size = _power(exps[table])
    x = (x.view(*size.shape, BLOCK, x.shape[-1]) * size[..., None, None]).view_as(x).transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[-1])


def _softmax_sums(scores, visible, v):
    """sum of softmax(scores) v over the visible positions and log-sum-exp; a row that sees nothing gives zeros."""
    scores = scores.masked_fill_(~visible, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1)
    p = p.div_(torch.where(total > 0, total, torch.ones_like(total)))
    return p @ v, lse


def _bent(s, case, scores, distance):
    """Cap and distance bias on scores [..., heads in a group, ...]; `distance` and the slopes broadcast to them."""
    scores = scores.mul_(s["scale"])
    if case["cap"]:
        scores = scores.div_(case["cap"]).tanh_().mul_(case["cap"])
    if s["slopes"] is not None:
        slopes = s["slopes"].view(1, case["kv_heads"], -1, 1, 1)
        scores = scores.sub_(slopes * distance)
    return scores


def _decode8(s, case):
    D, H, G = case["dim"], case["heads"], case["kv_heads"]
    k, v = _values(s["k_pages"], s["k_exps"], s["table"]), _values(s["v_pages"], s["v_exps"], s["table"])
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
    out, lse = _softmax_sums(scores, visible.view(B, 1, 1, S), v)
    return [out.reshape(B, H, D).to(s["q"].dtype), lse.reshape(B, H)]


def _prefill8(s, case):
    D, H, G = case["dim"], case["heads"], case["kv_heads"]
    k, v = _values(s["k_pages"], s["k_exps"], s["table"]), _values(s["v_pages"], s["v_exps"], s["table"])
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
    out, lse = _softmax_sums(scores, visible.view(B, 1, 1, T, S), v.unsqueeze(2))
    out = out.permute(0, 3, 1, 2, 4).reshape(B, T, H, D)[b, i]
    return [out.to(s["q"].dtype), lse.permute(0, 3, 1, 2).reshape(B, T, H)[b, i]]


# ---- the definition in 64 bits, one sequence at a time

def exact(case, seed):
    if case["op"] == "plan":
        return None  # whole numbers: nothing is computed
    s = prepare(case, seed)
    D, H, G, P = case["dim"], case["heads"], case["kv_heads"], case["page"]
    R = H // G
    new, total = _lengths(case)
    starts = [sum(new[:b]) for b in range(len(new))]
    device = s["q"].device

    if case["op"] in ("norm", "append8"):
        rot, out, keys = case["rot"] or D, [], []
        for b, (t, n) in enumerate(zip(new, total)):
            at = torch.arange(n - t, n, device=device)
            tokens = slice(starts[b], starts[b] + t)
            axes = [at] if s["positions"] is None else [a[tokens].long() for a in s["positions"]]
            c, e, p0 = [], [], 0
            for a, count in zip(axes, _sections(case)):
                c.append(s["cos_sin"][a, p0:p0 + count, 0].double())
                e.append(s["cos_sin"][a, p0:p0 + count, 1].double())
                p0 += count
            turn = torch.complex(torch.cat(c, 1), torch.cat(e, 1))[:, None]

            def turned(x, weight):
                x = x.double()
                if case["normed"]:
                    x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + _EPS) * s[weight].double()
                if case["interleaved"]:
                    z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2).contiguous()) * turn
                    return torch.cat([torch.view_as_real(z).reshape(*x.shape[:-1], rot), x[..., rot:]], -1)
                z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
                return torch.cat([z.real, z.imag, x[..., rot:]], -1)

            out.append(turned(s["q"][tokens], "q_weight"))
            keys.append(turned(s["k"][tokens], "k_weight"))
        if case["op"] == "append8":
            return [torch.cat(out), None, None, None, None]  # (what the codes are off the values is the format's, not the call's)
        k_pages = s["k_pages"].double()
        for b, (t, n) in enumerate(zip(new, total)):
            at = torch.arange(n - t, n, device=device)
            k_pages[s["table"][b].long()[at // P], :, at % P] = keys[b]
        return [torch.cat(out), k_pages, None]

    def rows(pages, exps, b, n):  # [G, n, D]
        used = s["table"][b, :(n + P - 1) // P].long()
        codes = pages.view(torch.uint8)[used].view(torch.float8_e4m3fn).double()
        size = torch.exp2(exps[used].double() - 127).repeat_interleave(BLOCK, dim=2)
        return torch.cat(list(codes * size[..., None]), dim=1)[:, :n]

    outs, lses = [], []
    slopes = None if s["slopes"] is None else s["slopes"].double()
    if case["op"] == "decode8":
        first, end = [0] * len(total), list(total)
    else:
        first, end = _visible(case)
    for b, (t, n) in enumerate(zip(new, total)):
        k, v = rows(s["k_pages"], s["k_exps"], b, n), rows(s["v_pages"], s["v_exps"], b, n)
        tokens = slice(starts[b], starts[b] + t)
        lo = torch.tensor(first[tokens], device=device)[:, None]
        hi = torch.tensor(end[tokens], device=device)[:, None]
        at = torch.arange(n - t, n, device=device)[:, None]
        j = torch.arange(n, device=device)[None]
        hidden = (j < lo) | (j >= hi)
        if case["window"]:
            hidden = hidden | (j <= at - case["window"])
        out = torch.zeros(t, H, D, dtype=torch.float64, device=device)
        lse = torch.zeros(t, H, dtype=torch.float64, device=device)
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
        outs.append(out)
        lses.append(lse)
    return [torch.cat(outs), torch.cat(lses)]
