"""MXFP4 blocks whose scale is so large that some of their elements are numbers and others infinities (2^126: 6 and 4 are; 2^127: 2 and more), beside those that
are all numbers (2^125) or NaN: every row that does not see them stays as it is, and so does every dimension beside them, finite places included."""
import math

import pytest
import torch

from paper_2508_19263_amd import zc
from tests.paged import starts
from tests.paged4 import MX, Cache4, values4
from tests.test_gpu_attend import check

pytestmark = pytest.mark.gpu

HALF, SIX = 1, 7                                               # codes of 0.5 and 6


def largest(cache):
    """The cache's numbers as 32 bits hold them."""
    for name in "kv":
        x = getattr(cache, name)
        setattr(cache, name, torch.where(x.abs() >= 2.0 ** 128, x.sign() * math.inf, x))
    return cache


def block(c, name, head, token, i, scale, codes):
    """Sets block i of a token: its scale, and codes of its 32 elements."""
    c.blocks[name][0, head, token, i] = scale
    code = torch.tensor([codes(e) for e in range(32)], dtype=torch.uint8, device="cuda")
    c.bits[name][0, head, token, i * 16:(i + 1) * 16] = code[0::2] | code[1::2] << 4


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_len", [1, 3, 40, 200])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 2), (7, 0)])
def test_values(dim, q_len, window, sinks):
    """With a scale of 0 every token that is seen weighs the same, so finite places are means of what is seen: at most 2^124 + 2^125 + 2^126 of 2^128 are added up."""
    last = dim // 32 - 1

    def edit(c):
        block(c, "v", 0, 299, 0, 253, lambda e: SIX if e in (3, 20) else HALF | 8 * (e & 1))
        block(c, "v", 0, 298, last, 254, lambda e: SIX | 8 if e == 9 else HALF)
        block(c, "v", 0, 290, last, 253, lambda e: SIX if e == 31 else HALF)
        block(c, "v", 0, 250, last, 252, lambda e: HALF | 8)
        block(c, "v", 1, 150, 0, 254, lambda e: SIX if e % 5 == 0 else 0)
        block(c, "v", 1, 296, last, 255, lambda e: HALF)
    q, out, lse = check(largest(Cache4([300], 2, dim, MX, edit=edit, scales=False)), [q_len], 4, window, sinks, scale=0.0)
    assert bool(lse.isfinite().all()) and bool(out[-1, 0, 3].isinf())
    if q_len == 200 and window == 7:
        assert bool(out[:40].isfinite().all())


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_len", [1, 3, 40, 200])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 2)])
def test_keys(dim, q_len, window, sinks):
    """One infinite element: the token's logit is an infinity of the query's sign; minus infinity has no weight, infinity leaves no number."""
    def edit(c):
        for token, scale in ((299, 253), (298, 254), (250, 254)):
            block(c, "k", 0, token, token % (dim // 32), scale, lambda e: SIX if e == token % 32 else 0)
    check(largest(Cache4([300], 2, dim, MX, edit=edit, scales=False)), [q_len], 4, window, sinks)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scales", [False, True])
@pytest.mark.parametrize("length", [1, 77, 3000])
def test_read_back(dim, scales, length):
    """Every block scale there is, over all elements: element * scale * S in 32 bits, rounded to BF16."""
    def edit(c):
        n = c.blocks["k"].numel()
        for i, name in enumerate("kv"):
            c.blocks[name].view(-1).copy_((torch.arange(n, device="cuda") * 7 + 252 + i) % 256)
            c.bits[name].view(-1).copy_((torch.arange(n * 16, device="cuda") * 11 + 5 * i) % 256)
    cache = Cache4([length], 2, dim, MX, edit=edit, scales=scales)
    k, v = zc.read_kv(cache.paged, starts([length]), length)
    for name, got in (("k", k), ("v", v)):
        x = values4(cache.bits[name], cache.blocks[name], MX)[0, :, :length].to(torch.float32)         # (what 32 bits do not hold becomes an infinity)
        if scales:
            x = x * getattr(cache, name + "s")[0].view(-1, 1, 1)
        want = x.to(torch.bfloat16).transpose(0, 1)
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(got.nan_to_num(7.0, math.inf, -math.inf), want.nan_to_num(7.0, math.inf, -math.inf))
    assert length < 77 or (bool(k.isinf().any()) and bool(k.isnan().any()))
