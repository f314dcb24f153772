"""Plain 64-bit form of attention over a paged cache, one row at a time, and how far a kernel's result may be from it.

The bounds are derived, not fitted.  With u the unit roundoff of the element type (2^-11 fp16, 2^-8 bf16), A = sum p |v| and out =
sum p v (p the exact probabilities):
  * the result is rounded once: u |out|;
  * every probability, relative to the row's running maximum, is rounded to the element type: u of itself, or half a
    subnormal step (fp16: 2^-25, of numbers whose maximum is 1, so that the sum is at least 1 less the roundings): u A + 2^-24 sum |v|
    over what is seen;
  * fp32: a score s is off by at most E = (dim + 8) 2^-24 scale sum |q k| + 8 * 2^-24 (|s| + cap + slope distance), which turns p into
    p (1 + 2 E) with the sum's; products and joins add a few 2^-24 of A: 4 E A + 2^-18 A.
Twice their sum is asserted.
"""
import math

import torch

UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def gather(pages, table, b, n):
    """Rows [kv_heads, n, ...] of sequence b, in 64 bits."""
    if n == 0:
        return pages[:0].transpose(0, 1).reshape(pages.shape[1], 0, *pages.shape[3:]).double()
    page = pages.shape[2]
    used = table[b, :(n + page - 1) // page].long()
    x = pages[used].transpose(0, 1)
    return x.reshape(x.shape[0], -1, *x.shape[3:])[:, :n].double()


def attend(q, k, v, at, lo, hi, scale, cap, slopes, window, dtype):
    """q [heads, dim] of one token at position `at`; k, v [kv_heads, n, dim]: (out, lse, p [heads, n], bound of out, bound of lse)."""
    H, D = q.shape
    G, n = k.shape[0], k.shape[1]
    u = UNIT[dtype]
    q = q.double()
    j = torch.arange(n, device=q.device)
    seen = (j >= lo) & (j < hi)
    if window:
        seen = seen & (j > at - window)
    kk, vv = k.repeat_interleave(H // G, 0), v.repeat_interleave(H // G, 0)
    kk = torch.where(seen[None, :, None], kk, torch.zeros_like(kk))
    vv = torch.where(seen[None, :, None], vv, torch.zeros_like(vv))
    s = (kk * q[:, None]).sum(-1) * scale
    size = (kk.abs() * q.abs()[:, None]).sum(-1) * abs(scale)
    if cap:
        s = cap * torch.tanh(s / cap)
    far = torch.zeros_like(s)
    if slopes is not None:
        far = slopes.double()[:, None] * (at - j).abs()[None]
        s = s - far
    s = s.masked_fill(~seen[None], -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None])
    out = (p[:, :, None] * vv).sum(1)
    A = (p[:, :, None] * vv.abs()).sum(1)
    finite = torch.where(seen[None], (D + 8) * 2.0 ** -24 * size + 8 * 2.0 ** -24 * (size.clamp(max=cap or math.inf) + cap + far.abs()),
                         torch.zeros_like(s))
    E = finite.max(-1).values if n else torch.zeros(H, device=q.device, dtype=torch.float64)
    bound = 2 * (u * out.abs() + (u + 2.0 ** -18 + 4 * E[:, None]) * A + 2.0 ** -24 * vv.abs().sum(1))
    lse_bound = 2 * (E + 2.0 ** -18 + 2.0 ** -22 * lse.abs().nan_to_num(0, 0, 0))
    return out, lse, p, bound, lse_bound, E
