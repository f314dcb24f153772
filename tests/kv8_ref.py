"""Plain forms of a cache held in 8 bits: what codes stand for, and what an append leaves, in 64 bits, one block at a time."""
import math

import torch

BLOCK = 16
LEAST = 10
TOP = {torch.float16: 127 + 8, torch.bfloat16: 127 + 120}  # the exponent of blocks that reach the end of the type
# from here on a value is an infinity in the type (half a step above its largest)
INFINITE = {torch.float16: 65520.0, torch.bfloat16: 2.0 ** 128 - 2.0 ** 119}


def decode(codes, exps):
    """Values of codes [..., positions, dim] with exponents [..., positions / 16], in 64 bits."""
    size = torch.exp2(exps.double() - 127).repeat_interleave(BLOCK, -1)
    return codes.view(torch.uint8).view(torch.float8_e4m3fn).double() * size[..., None]


def exponent(x, dtype):
    """Of a block of values, in 64 bits: the least e >= 10 with max |x| <= 448 * 2^(e - 127), over what is finite in the type."""
    x = x[x.abs() < INFINITE[dtype]]
    most = float(x.abs().max()) if x.numel() else 0.0
    if most == 0.0:
        return LEAST
    part, e = math.frexp(most)
    return max(e - 9 + (part > 0.875) + 127, LEAST)


def encode(x, e, dtype):
    """The nearest codes (ties to the even one) of x / 2^(e - 127), as bytes."""
    y = x * 2.0 ** (127 - e)
    end = 240.0 if e == TOP[dtype] else 448.0
    y = torch.where(x.abs() < INFINITE[dtype], y.clamp(-end, end), torch.full_like(y, math.nan))
    # (64 bits to 32 would round twice: only a tie could be hurt, and what is a tie in 32 bits and none in 64 is moved off it)
    f = y.float()
    near = torch.nextafter(f, torch.where(f.double() < y, math.inf, -math.inf).float())
    code = f.to(torch.float8_e4m3fn)
    tie = (f.double() != y) & (f.double() * 2 == (code.double() + near.to(torch.float8_e4m3fn).double()))
    return torch.where(tie, near.to(torch.float8_e4m3fn).view(torch.uint8), code.view(torch.uint8))


def append(codes, exps, x, begin, dtype):
    """Writes x [n, dim] as positions begin .. of one head of one sequence: codes [positions, dim] bytes, exps [positions / 16]."""
    n = x.shape[0]
    for block in range(begin // BLOCK, (begin + n - 1) // BLOCK + 1):
        lo, hi = max(begin, block * BLOCK), min(begin + n, (block + 1) * BLOCK)
        new = x[lo - begin:hi - begin]
        e = exponent(new, dtype)
        if block * BLOCK < begin:
            before = int(exps[block])
            if e > before:
                old = codes[block * BLOCK:begin].view(torch.float8_e4m3fn).double() * 2.0 ** (before - e)
                codes[block * BLOCK:begin] = old.float().to(torch.float8_e4m3fn).view(torch.uint8)
            e = max(e, before)
        exps[block] = e
        codes[lo:hi] = encode(new, e, dtype)


def turned(x, positions, cos_sin, sections, interleaved):
    """x [tokens, heads, dim] in 64 bits; positions [axes][tokens]; also how far a 32-bit form may be off, per token and head."""
    pairs = cos_sin.shape[1]
    rot = 2 * pairs
    axis = torch.tensor(sum([[a] * n for a, n in enumerate(sections)], []), device=x.device)
    p = torch.stack([q.long() for q in positions])[axis].t()  # [tokens, pairs]
    cs = cos_sin.double()[p, torch.arange(pairs, device=x.device)][:, None]
    c, s = cs[..., 0], cs[..., 1]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * s, a * s + b * c
    else:
        a, b = x[..., :pairs], x[..., pairs:rot]
        y[..., :pairs], y[..., pairs:rot] = a * c - b * s, a * s + b * c
    return y


def normed(x, weight, eps):
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    return y if weight is None else y * weight.double()
