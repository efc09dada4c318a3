"""Eviction where page offsets pass 32 bits, on the side that is read and on the side that is written."""
import pytest
import torch

from paper_2508_19263_amd import zc
from tests.paged import JUNK, Cache, gen

pytestmark = pytest.mark.gpu

BF16, E4M3 = zc.FMT_BF16, zc.FMT_FP8_E4M3


@pytest.mark.parametrize("fmt", [BF16, E4M3])
def test_eviction_from_and_to_pages_whose_offsets_pass_32_bits(fmt):
    cache = Cache([500, 37], 2, 128, fmt)
    w = torch.rand((2, 2, cache.paged.capacity), generator=gen(2), device="cuda")
    into = Cache([0, 0], 2, 128, fmt, room=100)
    pages = (cache.paged.k_pages, cache.paged.v_pages)
    room = (into.paged.k_pages, into.paged.v_pages)
    page_bytes = pages[0][0].numel() * pages[0].element_size()
    n = (1 << 32) // page_bytes + max(pages[0].shape[0], room[0].shape[0]) + 7

    def refill():
        for x in room:
            x.fill_(JUNK[fmt])

    refill()
    near = zc.evict(cache.paged, w, 90, into.paged)
    want = [x.clone() for x in room]
    assert not torch.equal(want[0], torch.full_like(want[0], JUNK[fmt])) and not torch.equal(want[0], want[1])
    refill()
    pools = []
    for x in pages:
        pool = torch.full((n,) + tuple(x.shape[1:]), JUNK[fmt], dtype=x.dtype, device="cuda")
        pool[-x.shape[0]:] = x
        pools.append(pool)
    far = zc.PagedCache(pools[0], pools[1], (cache.table + (n - pages[0].shape[0])).contiguous(), cache.lengths, fmt, cache.ks, cache.vs)
    kept = zc.evict(far, w, 90, into.paged)
    assert torch.equal(kept, near) and all(torch.equal(x, y) for x, y in zip(room, want))
    for pool in pools:
        pool.fill_(JUNK[fmt])
    away = zc.PagedCache(pools[0], pools[1], (into.table + (n - room[0].shape[0])).contiguous(), into.lengths, fmt)
    kept = zc.evict(cache.paged, w, 90, away)
    assert torch.equal(kept, near)
    for pool, y in zip(pools, want):
        assert torch.equal(pool[-y.shape[0]:], y) and bool((pool[:-y.shape[0]] == JUNK[fmt]).all())
