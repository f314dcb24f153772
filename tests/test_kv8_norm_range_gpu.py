"""Norms in an append to an 8-bit cache where factors leave what 32 bits hold although no result does: keys of zero and far below the root
of a small eps, weights near the end of bf16.  Results against the plain 64-bit form that the other appends are held to."""
import pytest
import torch

import kv8_ref as ref
import paper_2511_11248_amd as tman
from gpu_helpers import dev
from test_kv8_append_gpu import F32, Cache8, angles, check

pytestmark = pytest.mark.gpu
EPS = [1.1920929e-7, 1e-8, 1e-30]


def rule_of(dim, turned):
    return (angles(64, dim // 2), (dim // 4,), False) if turned else None


@pytest.mark.parametrize("eps", EPS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_blocks_of_zero_keys(eps, dim, turned, dtype):
    """Zero is its own norm: codes of zero and the least exponent, as a 16-bit cache would hold zeros."""
    C = Cache8(dim, [40], 4, 2, dim, 16, dtype)

    def edit(k, v):
        k[0:32] = 0

    check(C, [40], norm=tman.HeadNorm(None, 1 + torch.rand(dim, device=dev()), eps), rule=rule_of(dim, turned), edit=edit)
    for h in range(2):
        assert bool(((C.head(C.k, 0, h, 40)[:32] & 127) == 0).all())
        assert C.head(C.ke, 0, h, 40)[:2].tolist() == [ref.LEAST] * 2


@pytest.mark.parametrize("eps", EPS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("turned", [False, True])
def test_a_zero_token_that_opens_a_block_and_one_that_joins_it(eps, dim, turned):
    C = Cache8(dim + 1, [64], 2, 1, dim, 32, torch.float16)
    norm, zero = tman.HeadNorm(None, None, eps), lambda k, v: k.zero_()

    def step(n, edit=None):
        C.lens_list = [n]
        C.lens.copy_(C.ints([n]))
        check(C, [1], norm=norm, rule=rule_of(dim, turned), edit=edit, starts=n % 2 == 0)

    step(17, zero)   # opens a block
    assert bool(((C.head(C.k, 0, 0, 17)[16] & 127) == 0).all()) and int(C.head(C.ke, 0, 0, 17)[1]) == ref.LEAST
    step(18)         # an ordinary key behind it
    older, size = C.head(C.k, 0, 0, 18)[16:18], int(C.head(C.ke, 0, 0, 18)[1])
    step(19, zero)   # and zeros again: nothing of the block changes
    assert torch.equal(C.head(C.k, 0, 0, 19)[16:18], older) and int(C.head(C.ke, 0, 0, 19)[1]) == size
    assert bool(((C.head(C.k, 0, 0, 19)[18] & 127) == 0).all())


@pytest.mark.parametrize("eps", EPS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("size", [2.0 ** -133, 1e-38, 1e-30, 1e-12])
def test_keys_far_below_the_root_of_eps(eps, dim, turned, size):
    """x / sqrt(eps), however small: bf16's smallest numbers among them (2^-133)."""
    C = Cache8(dim + 2, [50], 2, 2, dim, 16, torch.bfloat16)

    def edit(k, v):
        k.sign_().mul_(size)

    check(C, [50], norm=tman.HeadNorm(None, 1 + torch.rand(2, dim, device=dev()), eps), rule=rule_of(dim, turned), edit=edit)
    assert not bool(torch.isnan(ref.decode(C.head(C.k, 0, 0, 50)[None], C.head(C.ke, 0, 0, 50)[None])[0, :50]).any())


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("weight", [2.0 ** 110, 2.0 ** -100])
@pytest.mark.parametrize("size", [2.0 ** 59, 2.0 ** 8, 1.0, 2.0 ** -8])
def test_weights_that_a_large_or_small_key_would_take_out_of_fp32(dim, turned, weight, size):
    """The normed key times the weight is a number of bf16, in whatever order it is made."""
    C = Cache8(dim + 3, [20], 2, 1, dim, 16, torch.bfloat16)

    def edit(k, v):
        k.clamp_(-2, 2).mul_(size)

    w = torch.full((dim,), weight, device=dev())
    check(C, [20], norm=tman.HeadNorm(None, w, 1e-20), rule=rule_of(dim, turned), edit=edit, q=False)
    assert not bool(torch.isnan(ref.decode(C.head(C.k, 0, 0, 20)[None], C.head(C.ke, 0, 0, 20)[None])[0, :20]).any())


@pytest.mark.parametrize("eps", [1e-6, 1e30, 1e36, 3e38, torch.finfo(torch.float32).max])
def test_an_eps_beside_squares_that_leave_fp32(eps):
    """Rows of 1e19 to 3e38 and an eps of their squares' size, into either cache."""
    x = torch.zeros(4, 3, 64, dtype=torch.bfloat16, device=dev())
    for i, size in enumerate((1e18, 3e18, 1e19, 3e38)):
        x[i] = size
    x[:, :, ::3] *= -0.5
    pages = torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16, device=dev())
    table, lens = torch.arange(4, dtype=torch.int32, device=dev())[:, None].contiguous(), torch.ones(4, dtype=torch.int32, device=dev())
    out = torch.empty(4, 1, 64, dtype=torch.bfloat16, device=dev())
    norm = tman.HeadNorm(None, None, eps)
    tman.tman_norm_rope_append(tman.KvCache(pages, torch.zeros_like(pages), table), norm, x[:, :1], x[:, 1:2], x[:, 2:], lens, out)
    want = ref.normed(x.double(), None, float(torch.tensor(eps, dtype=torch.float32)))
    for got, h in ((out[:, 0], 0), (pages[:, 0, 0], 1)):
        assert bool(((got.double() - want[:, h]).abs() <= (2.0 ** -8 + F32) * want[:, h].abs()).all())
    codes, exps = torch.zeros(4, 1, 16, 64, dtype=torch.uint8, device=dev()), torch.zeros(4, 1, 1, dtype=torch.uint8, device=dev())
    cache = tman.KvCache8(codes, torch.zeros_like(codes), exps, torch.zeros_like(exps), table, torch.bfloat16)
    tman.tman_kv8_append(cache, x[:, :1], x[:, 1:2], x[:, 2:], lens, out, norm=norm)
    got = ref.decode(codes, exps)[:, 0, 0]
    assert bool(((got - want[:, 1]).abs() <= (2.0 ** -4 + F32) * want[:, 1].abs()).all())
    assert bool(((out[:, 0].double() - want[:, 0]).abs() <= (2.0 ** -8 + F32) * want[:, 0].abs()).all())
