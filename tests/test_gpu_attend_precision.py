"""Attention over K/V pages where numbers lie far apart or are none, against its definition in 64 bits (tests/paged.py)."""
import math

import pytest
import torch

from paper_2508_19263_amd import zc
from tests.paged import Cache, agree, attention, gen, starts, stored
from tests.test_gpu_attend import check, queries

pytestmark = pytest.mark.gpu

BF16, E4M3, E5M2 = zc.FMT_BF16, zc.FMT_FP8_E4M3, zc.FMT_FP8_E5M2


@pytest.mark.parametrize("fmt", [BF16, E4M3, E5M2])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nats", [17.0, 20.0])
@pytest.mark.parametrize("q_len,length", [(1, 600), (1, 9000), (30, 600), (150, 600)])
def test_many_light_tokens_beside_a_heavy_one(fmt, dim, nats, q_len, length):
    """The first token's logit lies `nats` above the others' and its value is zero: the result is the others' alone.

    The tolerance of attention() is relative to each weight.  Half precision also has a smallest number, 2^-24: with weights lifted by
    2^7, of which the heaviest is at least 1 before, one is off by up to 2^-25 2^-7 of the heaviest, so out by 2^-32 sum |v|, doubled as there."""
    def edit(c):
        c.k[..., 0] = 0
        c.k[:, :, 0] = 0
        c.k[:, :, 0, 0] = stored(torch.full(c.k.shape[:2], 16.0, device="cuda"), fmt)
        c.v[:] = stored(50 * torch.randn(c.v.shape, generator=gen(7), device="cuda").abs(), fmt)
        c.v[:, :, 0] = 0
    cache = Cache([length], 1, dim, fmt, edit=edit, scales=False)
    q = (queries(q_len, 2, dim).float() * 0.05)
    q[..., 0] = nats / (16.0 * dim ** -0.5)
    q = q.to(torch.bfloat16)
    out, lse = zc.attend(q, cache.paged, q_start=starts([q_len]), max_q_len=q_len)
    want, want_lse, _, tol, tol_lse, _ = attention(q, [q_len], cache)
    floor = 2 * 2.0 ** -32 * cache.rows("v", 0, 0).abs().sum(dim=0) if fmt != BF16 else 0.0
    agree(out, want, tol + floor, "out")
    agree(lse, want_lse, tol_lse, "lse")


@pytest.mark.parametrize("lens,q_lens", [([300, 2], [1, 5]), ([300, 20], [1, 40]), ([3000, 2], [1, 5]), ([3000, 900], [1, 1])])
@pytest.mark.parametrize("fmt", [BF16, E4M3])
def test_a_scale_that_is_not_a_number(fmt, lens, q_lens):
    """It is seen in its head's results and weights, and nowhere else; queries that see nothing have nothing to do with it."""
    cache = Cache(lens, 2, 128, fmt, scales=True)
    q, w = queries(sum(q_lens), 8, 128), torch.zeros((2, 2, cache.paged.capacity), device="cuda")
    more = dict(q_start=starts(q_lens), max_q_len=max(q_lens))
    want, want_lse = zc.attend(q, cache.paged, weights_out=w, **more)
    cache.ks[1, 0] = float("nan")
    w_nan = torch.zeros_like(w)
    out, lse = zc.attend(q, cache.paged, weights_out=w_nan, **more)
    blind, first = max(0, q_lens[1] - lens[1]), q_lens[0]        # query tokens of the second sequence that see nothing
    hit = torch.zeros((sum(q_lens), 8), dtype=torch.bool, device="cuda")
    hit[first + blind:, :4] = True
    assert bool(out[hit].isnan().all()) and bool(lse[hit].isnan().all())
    assert torch.equal(out[~hit], want[~hit]) and torch.equal(lse[~hit], want_lse[~hit])
    assert blind == 0 or (not bool(out[first:first + blind].any()) and bool((lse[first:first + blind] == -math.inf).all()))
    assert bool(w_nan[1, 0, :lens[1]].isnan().all())
    w_nan[1, 0], w[1, 0] = 0, 0
    assert torch.equal(w_nan, w)


@pytest.mark.parametrize("answers", [2, 40])
def test_a_prefixs_scale_that_is_not_a_number(answers):
    """Answers that the window has led away from the prefix do not see it."""
    cache = Cache([50] + [3] * (answers - 1), 2, 128, E4M3)
    prefix = Cache([300], 2, 128, E4M3, seed=3)
    q = queries(answers, 8, 128)
    want, want_lse = zc.attend_shared(q, prefix.paged, cache.paged, window=10)
    prefix.ks[0, 0] = float("nan")
    out, lse = zc.attend_shared(q, prefix.paged, cache.paged, window=10)
    assert bool(out[1:, :4].isnan().all()) and bool(lse[1:, :4].isnan().all())
    for got, there in ((out, want), (lse, want_lse)):
        assert torch.equal(got[0], there[0]) and torch.equal(got[:, 4:], there[:, 4:])


@pytest.mark.parametrize("q_lens", [[1, 7], [1, 70]])
def test_a_scale_of_zero_with_large_keys(q_lens):
    """Products around 1e32 and a factor of 0: every token has the same weight."""
    def edit(c):
        c.k[:] = stored(c.k.view(torch.bfloat16).float() * 1e30, BF16)
    check(Cache([300, 41], 2, 128, BF16, edit=edit), q_lens, 4, scale=0.0, weights=True)


@pytest.mark.parametrize("fmt", [BF16, E4M3, E5M2])
@pytest.mark.parametrize("q_len,length", [(1, 600), (1, 9000), (150, 600)])
def test_logits_whose_rounding_is_as_large_as_they_lie_apart(fmt, q_len, length):
    """All logits lie around 2^25 in base 2, where numbers in 32 bits are 4 apart, and the later tokens' 8 above the first ones': the weights'
    exponents are off by up to 2, and no weight may leave its type's range for it."""
    def edit(c):
        c.k[:] = 0
        c.k[..., 0] = stored(torch.full(c.k.shape[:3], 16.0, device="cuda"), fmt)
        c.k[:, :, 256:, 1] = stored(torch.ones(c.k.shape[:2] + (c.k.shape[2] - 256,), device="cuda"), fmt)
    cache = Cache([length], 1, 128, fmt, edit=edit, scales=False)
    q = torch.zeros((q_len, 2, 128), dtype=torch.bfloat16, device="cuda")
    q[..., 0], q[..., 1] = 1.0, 2.0 ** -18
    for scale in (1453600.0, 1453500.0, 1400000.0, 2907000.0):
        out, lse = zc.attend(q, cache.paged, q_start=starts([q_len]), max_q_len=q_len, scale=scale)
        want, want_lse, _, tol, tol_lse, _ = attention(q, [q_len], cache, scale=scale)
        agree(out, want, tol, "out")
        agree(lse, want_lse, tol_lse, "lse")
        assert float(out.abs().max()) <= 1.01 * float(cache.rows("v", 0, 0).abs().max())
