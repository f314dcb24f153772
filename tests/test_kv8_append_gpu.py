"""Appends with norms, and to a cache held in 8 bits, against plain 64-bit forms: what the codes are, whose power of two it is, older
positions of a block, values at the ends of the types, what must stay as it was."""
import math

import pytest
import torch

import kv8_ref as ref
import paper_2511_11248_amd as tman
from attention_ref import UNIT
from gpu_helpers import dev

pytestmark = pytest.mark.gpu
ERR_INDEX = -10
NAN, INF = float("nan"), float("inf")
# A 32-bit norm and rotation: 24 roundings of the sum of squares and 6 more at most (2^-24 each, the sum's as its mean), the reciprocal
# root 2^-23, cos and sin are inputs.  Of the head's largest magnitude.
F32 = 2.0 ** -19


class Cache8:
    """Sequences of given lengths; every byte of the pool and every exponent starts as garbage of its own."""

    def __init__(self, seed, lens, heads, kv_heads, dim, page, dtype, extra=2):
        self.gen = torch.Generator(device=dev())
        self.gen.manual_seed(seed)
        self.lens_list, self.heads, self.kv_heads, self.dim, self.page, self.dtype = list(lens), heads, kv_heads, dim, page, dtype
        wide = max(1, max((n + page - 1) // page for n in lens)) + 1
        n_pages = sum((n + page - 1) // page for n in lens) + extra
        order = torch.randperm(n_pages, generator=self.gen, device=dev()).tolist()
        shape = (n_pages, kv_heads, page, dim)
        self.k, self.v = self.bytes(*shape), self.bytes(*shape)
        self.ke, self.ve = self.bytes(*shape[:2], page // 16), self.bytes(*shape[:2], page // 16)
        table = torch.full((len(lens), wide), 2 ** 30, dtype=torch.int32)
        for b, n in enumerate(lens):
            for i in range((n + page - 1) // page):
                table[b, i] = order.pop()
        self.table, self.lens = table.to(dev()), self.ints(lens)
        self.cache = tman.KvCache8(self.k, self.v, self.ke, self.ve, self.table, dtype)

    def bytes(self, *shape):
        return torch.randint(0, 256, shape, generator=self.gen, device=dev(), dtype=torch.uint8)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.gen, device=dev())

    def ints(self, x):
        return torch.tensor(x, dtype=torch.int32, device=dev())

    def head(self, pages, b, h, n):
        """Rows of a head of sequence b up to position n (whole pages), copied."""
        used = self.table[b, :(n + self.page - 1) // self.page].long()
        return pages[used, h].reshape(-1, *pages.shape[3:]).clone()

    def put(self, pages, b, h, rows):
        used = self.table[b, :rows.shape[0] // (pages.shape[2])].long()
        pages[used, h] = rows.view(-1, *pages.shape[2:])


def angles(n_pos, rot):
    pos = torch.arange(n_pos, dtype=torch.float64, device=dev())
    freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=dev()) / rot)
    a = pos[:, None] * freq[None]
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def near_border(x, dtype):
    """Whether a block's largest value is where 32 bits may choose the other exponent."""
    x = x[x.abs() < ref.INFINITE[dtype]]
    part = math.frexp(float(x.abs().max()))[0] if x.numel() else 0.5
    return abs(part - 0.875) < 4 * F32


def check(C, new, rule=None, norm=None, positions=None, starts=True, q=True, magnitude=1.0, edit=None):
    """One append of new[b] tokens to each sequence; compares everything that it writes, and everything that it does not."""
    B, H, G, D, dtype = len(C.lens_list), C.heads, C.kv_heads, C.dim, C.dtype
    N = sum(new)
    qkv = (C.normal(N, H + 2 * G, D) * magnitude).to(dtype)
    if edit:
        edit(qkv[:, H:H + G], qkv[:, H + G:])
    k, v = qkv[:, H:H + G], qkv[:, H + G:]
    out = torch.full((N, H + 1, D), 7.0, dtype=dtype, device=dev())[:, :H]
    q_start = [sum(new[:b]) for b in range(B + 1)]
    before = [t.clone() for t in (C.k, C.v, C.ke, C.ve)]
    tman.tman_kv8_append(C.cache, qkv[:, :H] if q else None, k, v, C.lens, out if q else None, norm=norm,
                         rope=None if rule is None else tman.Rope(*rule), positions=positions,
                         q_start=C.ints(q_start) if starts else None)
    assert tman.tman_device_status() == 0

    at = torch.cat([torch.arange(n - t, n) for n, t in zip(C.lens_list, new)]).to(dev())
    def made(x, weight):
        y = x.double()
        if norm is not None:
            y = ref.normed(y, weight, norm.eps)
        if rule is not None:
            cs, sections, interleaved = rule
            y = ref.turned(y, positions if positions is not None else [at] * len(sections), cs, sections, interleaved)
        return y

    if q:
        want = made(qkv[:, :H], None if norm is None else norm.q_weight)
        off = (out.double() - want).abs()
        bound = UNIT[dtype] * want.abs() + F32 * want.abs().amax(-1, keepdim=True) + (2.0 ** -25 if dtype == torch.float16 else 0)
        assert bool((off <= bound * (1 + 2.0 ** -10)).all())
    keys, values = made(k, None if norm is None else norm.k_weight), v.double()
    for pages, exps, old_pages, old_exps, x, exact in ((C.v, C.ve, before[1], before[3], values, True),
                                                       (C.k, C.ke, before[0], before[2], keys, rule is None and norm is None)):
        for b, (n, t) in enumerate(zip(C.lens_list, new)):
            for h in range(G if t else 0):
                got, got_e = C.head(pages, b, h, n), C.head(exps, b, h, n)
                want, want_e = C.head(old_pages, b, h, n).cpu(), C.head(old_exps, b, h, n).cpu()
                rows = x[q_start[b]:q_start[b + 1], h].cpu()
                ref.append(want, want_e, rows, n - t, dtype)
                if exact:
                    nan = (want & 127) == 127
                    assert torch.equal(got_e.cpu(), want_e)
                    assert torch.equal(got.cpu() & ~(nan * 128).to(torch.uint8), want & ~(nan * 128).to(torch.uint8))
                    continue
                # older rows follow from the exponents; new ones are within half a step of their codes, and 32 bits' error
                for block in range((n - t) // 16, (n - 1) // 16 + 1):
                    lo, hi = max(n - t, block * 16), min(n, block * 16 + 16)
                    e = int(got_e[block])
                    part = rows[lo - n + t:hi - n + t]
                    if e != int(want_e[block]):
                        assert near_border(part, dtype) and abs(e - int(want_e[block])) == 1
                        continue
                    assert torch.equal(got[block * 16:lo].cpu(), want[block * 16:lo])
                    y = ref.decode(got[lo:hi].cpu()[None], torch.full((1, 1), e, dtype=torch.uint8))[0, :hi - lo] if hi - lo == 16 else \
                        got[lo:hi].cpu().view(torch.float8_e4m3fn).double() * 2.0 ** (e - 127)
                    bound = torch.maximum(part.abs() * 2.0 ** -4, torch.tensor(2.0 ** (e - 127 - 10), dtype=torch.float64))
                    bound = bound + F32 * part.abs().nan_to_num(0.0).amax(-1, keepdim=True)
                    nan = torch.isnan(part)
                    assert torch.equal(torch.isnan(y), nan)
                    assert bool(((y - part).abs() <= bound)[~nan].all())
                got_rest, want_rest = got[n:].cpu(), want[n:]
                assert torch.equal(got_rest, want_rest)
                C.put(old_pages, b, h, got)
                C.put(old_exps, b, h, got_e)
            if exact:
                for h in range(G if t else 0):
                    C.put(old_pages, b, h, C.head(pages, b, h, n))
                    C.put(old_exps, b, h, C.head(exps, b, h, n))
        # all else is as it was
        assert torch.equal(pages, old_pages) and torch.equal(exps, old_exps)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads,page", [(4, 4, 16), (6, 2, 32), (8, 1, 64), (10, 5, 256)])
def test_fresh_prompts(dtype, dim, heads, kv_heads, page):
    new = [1, 0, 15, 16, 17, 33, 70]
    C = Cache8(dim + heads, new, heads, kv_heads, dim, page, dtype)
    check(C, new)
    check(C, new, rule=(angles(128, dim), (dim // 2,), False))


@pytest.mark.parametrize("dim", [64, 256])
def test_more_than_64_sequences(dim):
    """Blocks are found over groups of sequences, some of which have no tokens."""
    lens = [(31 * b * b) % 90 + 1 for b in range(150)]
    new = [0 if b % 6 == 2 else min(n, 1 + (11 * b) % 40) for b, n in enumerate(lens)]
    C = Cache8(dim, lens, 2, 1, dim, 16, torch.float16)
    for b, n in enumerate(lens):  # older positions are finite codes of sane exponents
        used = C.table[b, :(n + 15) // 16].long()
        for pages, exps in ((C.k, C.ke), (C.v, C.ve)):
            pages[used] = (C.normal(len(used), 1, 16, dim) * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            exps[used] = 119 + b % 3
    check(C, new, rule=(angles(128, dim), (dim // 2,), False))
    C.lens_list = [n for n in lens]
    check(C, [1] * 150, starts=False)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,rot,sections,interleaved", [(64, 64, (32,), False), (128, 64, (32,), True), (128, 128, (20, 24, 20), False),
                                                          (256, 16, (8,), False), (256, 256, (50, 78), True), (64, 48, (24,), False)])
@pytest.mark.parametrize("weights", ["none", "shared", "per head"])
def test_norms_and_rotations(dtype, dim, rot, sections, interleaved, weights):
    lens, new, H, G = [40, 300, 16, 129], [40, 33, 1, 64], 6, 3
    C = Cache8(rot + dim, lens, H, G, dim, 32, dtype)
    for b in range(4):  # older positions are finite codes of sane exponents
        used = C.table[b, :(lens[b] + 31) // 32].long()
        for pages, exps in ((C.k, C.ke), (C.v, C.ve)):
            pages[used] = (C.normal(len(used), G, 32, dim) * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            exps[used] = 120
    shape = {"none": None, "shared": (), "per head": (1,)}[weights]
    qw = kw = None
    if shape is not None:
        qw = 1 + 0.5 * C.normal(*((H, dim) if shape else (dim,)))
        kw = 1 + 0.5 * C.normal(*((G, dim) if shape else (dim,)))
    norm = tman.HeadNorm(qw, kw, 1e-6)
    positions = None
    if len(sections) > 1:
        positions = torch.randint(0, 500, (len(sections), sum(new)), generator=C.gen, device=dev(), dtype=torch.int32)
    check(C, new, rule=(angles(500, rot), sections, interleaved), norm=norm, positions=positions, magnitude=3.0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_single_tokens_that_grow_and_shrink(dtype, dim):
    """40 steps of three sequences: the powers of two of their blocks rise with the largest value, and older codes follow."""
    C = Cache8(dim, [1, 14, 31], 4, 2, dim, 32, dtype)
    longest = [n + 40 for n in C.lens_list]
    C = Cache8(dim, longest, 4, 2, dim, 32, dtype)
    C.lens_list = [1, 14, 31]
    C.lens.copy_(C.ints(C.lens_list))
    check(C, C.lens_list)
    for step in range(40):
        C.lens_list = [n + 1 for n in C.lens_list]
        C.lens.copy_(C.ints(C.lens_list))
        check(C, [1, 1, 1], starts=step % 2 == 0, q=step % 3 > 0, magnitude=4.0 ** ((step * 7) % 9 - 4))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_ends_of_the_types(dtype):
    top = torch.finfo(dtype).max
    tiny = torch.finfo(dtype).smallest_subnormal if hasattr(torch.finfo(dtype), "smallest_subnormal") else torch.finfo(dtype).tiny

    def edit(k, v):
        for x in (k, v):
            x[0:16] = 0                   # nothing but zeros
            x[16:32, :, 3] = top          # the largest value
            x[32:48, :, 5] = INF
            x[33, :, 6] = NAN
            x[34, :, 7] = -INF
            x[48:64] = INF                # nothing that is finite
            x[64:80] = tiny
            x[80:96, :, 0] = top * 0.875  # where the last exponent begins, and above
            x[81, :, 1] = top * 0.9
            x[96:112] = 1.75              # exactly the end of a power of two
            x[112:128] = 1.0
            x[113, :, 2] = 1.7578125      # and just above

    C = Cache8(5, [128], 2, 2, 64, 64, dtype)
    check(C, [128], edit=edit)
    used = C.table[0, :2].long()
    for pages, exps in ((C.k, C.ke), (C.v, C.ve)):
        x = ref.decode(pages[used], exps[used])
        finite = torch.isfinite(x.to(dtype))
        want = torch.ones(128, dtype=torch.bool, device=dev())
        rows = torch.cat([x[0], x[1]], 1)
        assert bool(torch.isfinite(rows[:, :32].to(dtype)).all()) and bool(torch.isfinite(rows[:, 64:].to(dtype)).all())
        assert bool(torch.isnan(rows[:, 48:64]).all()) and bool(torch.isnan(rows[:, 32:48, 5]).all())
        assert finite is not None and want is not None


@pytest.mark.parametrize("dim,rule", [(64, False), (128, False), (128, True), (256, True)])
def test_signalling_nan_beside_large_values(dim, rule):
    """Bits of bf16 may be signalling NaN: they are held as NaN, and the others as without them."""
    def edit(k, v):
        for x in (k, v):
            x[:, :, 0] = 300.0
            bits = x.view(torch.int16)
            bits[3, :, 1], bits[20, :, dim - 1], bits[33, 0, 2:9] = 0x7f81, -0x7f + 0x1, 0x7fa0  # 0x7f81, 0xff82, 0x7fa0

    C = Cache8(6, [40], 2, 2, dim, 16, torch.bfloat16)
    check(C, [40], edit=edit, rule=(angles(64, 16), (8,), False) if rule else None)


def test_norms_in_an_8_bit_append_of_values_whose_squares_leave_fp32():
    """Also where a weight would take the value itself out of fp32."""
    C = Cache8(7, [3], 2, 1, 64, 16, torch.bfloat16)
    w = torch.full((64,), 7.0, device=dev())

    def edit(k, v):
        k[0], k[1, :, :32], k[2] = 3e38, -2e25, 1e-3

    check(C, [3], norm=tman.HeadNorm(w, w, 1e-6), edit=edit, rule=(angles(64, 64), (32,), False))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_norms_of_rows_that_are_not_finite(dtype):
    def edit(k, v):
        k[3, :, 2], k[4, :, 7], k[20], k[21, :, 60] = INF, NAN, -INF, INF
        k[22] = 0

    C = Cache8(8, [30], 4, 2, 64, 16, dtype)
    check(C, [30], edit=edit, norm=tman.HeadNorm(None, 1 + torch.rand(64, device=dev()), 1e-6), rule=(angles(64, 32), (16,), True))


def test_growth_by_much_and_garbage_exponents():
    """A block whose older positions are far smaller: their codes vanish.  Exponents of blocks that nobody wrote do not matter."""
    C = Cache8(9, [33], 2, 1, 64, 16, torch.bfloat16)
    C.lens_list = [5]
    C.lens.copy_(C.ints([5]))
    check(C, [5], magnitude=1e-30)
    C.lens_list = [18]
    C.lens.copy_(C.ints([18]))
    check(C, [13], magnitude=1e30)
    C.lens_list = [33]
    C.lens.copy_(C.ints([33]))
    check(C, [15], magnitude=1.0)


def test_norms_of_values_whose_squares_leave_fp32():
    x = torch.zeros(2, 3, 64, dtype=torch.bfloat16, device=dev())
    x[0] = 1e30
    x[1, 0, :32], x[1, 1, 5], x[1, 2] = 3e38, -2e25, 1e-3
    pages = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16, device=dev())
    table, lens = torch.tensor([[0], [1]], dtype=torch.int32, device=dev()), torch.tensor([1, 1], dtype=torch.int32, device=dev())
    cache = tman.KvCache(pages, torch.zeros_like(pages), table)
    out = torch.empty(2, 1, 64, dtype=torch.bfloat16, device=dev())
    tman.tman_norm_rope_append(cache, tman.HeadNorm(None, None, 1e-6), x[:, :1], x[:, 1:2], x[:, 2:], lens, out)
    for got, h in ((out[:, 0], 0), (pages[:, 0, 0], 1)):
        want = ref.normed(x[:, h].double(), None, 1e-6)
        assert bool(((got.double() - want).abs() <= (2.0 ** -8 + F32) * want.abs()).all())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 6, 2), (128, 16, 16), (256, 5, 1)])
@pytest.mark.parametrize("many", [False, True])
def test_norms_into_a_16_bit_cache(dtype, dim, heads, kv_heads, many):
    gen = torch.Generator(device=dev())
    gen.manual_seed(dim)
    lens, new, page = ([5000, 3], [4500, 2], 64) if many else ([70, 1, 33], [1, 1, 1], 16)
    N, B = sum(new), len(lens)
    rot = dim // 2
    qkv = torch.randn(N, heads + 2 * kv_heads, dim, generator=gen, device=dev()).to(dtype)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    qw, kw = torch.randn(heads, dim, generator=gen, device=dev()), torch.randn(kv_heads, dim, generator=gen, device=dev())
    wide = (max(lens) + page - 1) // page
    kp = torch.full((wide * B, kv_heads, page, dim), 3.0, dtype=dtype, device=dev())
    vp = kp.clone()
    table = torch.arange(wide * B, dtype=torch.int32, device=dev()).flip(0).view(B, wide).contiguous()
    cs = angles(max(lens), rot)
    starts = [sum(new[:b]) for b in range(B + 1)]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev())  # noqa: E731
    weights = torch.full(kp.shape[:3], 5.0, device=dev())
    out = q if many else torch.empty(N, heads, dim, dtype=dtype, device=dev())
    at = torch.cat([torch.arange(n - t, n) for n, t in zip(lens, new)]).to(dev())
    want_q = ref.turned(ref.normed(q.double(), qw, 1e-5), [at], cs, (rot // 2,), False)
    want_k = ref.turned(ref.normed(k.double(), kw, 1e-5), [at], cs, (rot // 2,), False)
    tman.tman_norm_rope_append(tman.KvCache(kp, vp, table), tman.HeadNorm(qw, kw, 1e-5), q, k, v, ints(lens), out, rope=tman.Rope(cs),
                               q_start=ints(starts), weights=weights)
    assert tman.tman_device_status() == 0
    owner = torch.cat([torch.full((t,), b) for b, t in enumerate(new)]).to(dev())
    pages, slots = table[owner, at // page].long(), at % page
    for got, want in ((out, want_q), (kp[pages, :, slots], want_k)):
        bound = UNIT[dtype] * want.abs() + F32 * want.abs().amax(-1, keepdim=True) + (2.0 ** -25 if dtype == torch.float16 else 0)
        assert bool(((got.double() - want).abs() <= bound * (1 + 2.0 ** -10)).all())
    assert torch.equal(vp[pages, :, slots], v)
    assert bool((weights[pages, :, slots] == 0).all())
    rest = torch.ones(kp.shape[0], page, dtype=torch.bool, device=dev())
    rest[pages, slots] = False
    assert bool((kp.transpose(1, 2)[rest] == 3).all()) and bool((vp.transpose(1, 2)[rest] == 3).all())


def test_what_is_out_of_range_is_dropped_and_reported():
    C = Cache8(3, [20, 40], 2, 1, 64, 16, torch.float16)
    table = C.table.clone()
    C.table[0, 1] = 10 ** 6      # a page that the pool has not
    before = [t.clone() for t in (C.k, C.v, C.ke, C.ve)]
    kv = torch.randn(4, 2, 64, device=dev()).half()
    args = lambda lens, n: (C.cache, None, kv[:n, :1], kv[:n, 1:], C.ints(lens), None)  # noqa: E731
    tman.tman_kv8_append(*args([20, 40], 4), q_start=C.ints([0, 3, 3]))
    assert tman.tman_device_status() == ERR_INDEX and tman.tman_device_status() == 0
    C.table.copy_(table)
    tman.tman_kv8_append(*args([2 ** 31 - 1, 40], 2), q_start=C.ints([0, 2, 2]))
    assert tman.tman_device_status() == ERR_INDEX
    tman.tman_kv8_append(*args([0, -5], 2))
    assert tman.tman_device_status() == ERR_INDEX
    for was, now in zip(before, (C.k, C.v, C.ke, C.ve)):
        assert torch.equal(was, now)
    # more tokens than positions: those in front of position zero are dropped
    tman.tman_kv8_append(*args([2, 40], 4), q_start=C.ints([0, 4, 4]))
    assert tman.tman_device_status() == ERR_INDEX
    page = int(C.table[0, 0])
    got = ref.decode(C.v[page, 0][None], C.ve[page, 0][None])[0, :2]
    want = kv[2:4, 1].double()
    assert bool(((got - want).abs() <= (want.abs() * 2.0 ** -4).clamp(min=2.0 ** -10)).all())
