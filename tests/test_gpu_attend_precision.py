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
