"""Limits below the table's room, scratch of the caller's, mixed batches: against the definition in 64 bits (tests/paged.py)."""
import ctypes as C

import pytest
import torch

from paper_2508_19263_amd import zc
from tests.paged import Cache, gen, starts
from tests.test_gpu_attend import check, queries

pytestmark = pytest.mark.gpu

BF16, E4M3 = zc.FMT_BF16, zc.FMT_FP8_E4M3


@pytest.mark.parametrize("fmt,dim", [(BF16, 64), (E4M3, 128)])
@pytest.mark.parametrize("q_lens,lens", [([1, 1, 1], [999, 40, 0]), ([3, 1, 2], [999, 40, 17]), ([40, 3, 9], [999, 40, 17]), ([700, 3, 9], [1337, 40, 17]),
                                         ([1, 1, 1], [2999, 40, 1])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 5)])
def test_the_longest_length_below_the_tables_room(fmt, dim, q_lens, lens, window, sinks):
    """Few rows and many, weights from the logits and from the keys, and from parts of the rows: the weights lie by the table's room."""
    cache = Cache(lens, 2, dim, fmt, room=5000)
    check(cache, q_lens, 4, window, sinks, weights=True, max_kv_len=max(lens))
    check(cache, q_lens, 4, window, sinks, max_kv_len=max(lens))


@pytest.mark.parametrize("fmt,dim", [(BF16, 128), (E4M3, 64)])
@pytest.mark.parametrize("q_lens,lens", [([1, 1, 1], [199, 40, 0]), ([3, 1, 2], [199, 1, 17]), ([1] * 40, [7 + i for i in range(40)]), ([100, 3], [333, 9])])
@pytest.mark.parametrize("prefix", [37, 2001])
def test_limits_of_a_prefix_and_what_follows_it(fmt, dim, q_lens, lens, prefix):
    pre, cache = Cache([prefix], 2, dim, fmt, room=4000, seed=9), Cache(lens, 2, dim, fmt, room=700)
    for window, sinks in ((0, 0), (150, 5)):
        check(cache, q_lens, 4, window, sinks, prefix=pre, max_kv_len=max(lens), max_prefix_len=prefix)


@pytest.mark.parametrize("q_lens", [[2, 1], [90, 1]])
def test_lengths_above_a_limit_are_taken_as_the_limit(q_lens):
    cache, pre = Cache([900, 77], 2, 128, E4M3, room=2000), Cache([500], 2, 128, E4M3, room=1000, seed=4)
    q, w = queries(sum(q_lens), 8, 128), [torch.full((2, 2, cache.paged.capacity), -7.0, device="cuda") for _ in range(2)]
    more = dict(q_start=starts(q_lens), max_q_len=max(q_lens), window=400, sinks=3, max_kv_len=613)
    results = []
    for i, (own, prefix) in enumerate(((900, 500), (613, 301))):
        cache.lengths[0], pre.lengths[0] = own, prefix
        results.append(zc.attend(q, cache.paged, weights_out=w[i], **more) + zc.attend_shared(q, pre.paged, cache.paged, max_prefix_len=301, **more))
    assert all(torch.equal(a, b) for a, b in zip(*results)) and torch.equal(*w)
    assert bool((w[0][0, :, 613:] == -7).all()) and bool((w[0][0, :, :613] >= 0).all())


@pytest.mark.parametrize("fmt,dim", [(BF16, 64), (E4M3, 128)])
def test_weights_of_few_rows_with_room_for_more_logits_than_are_kept(fmt, dim):
    """Eight tables with room for a million tokens, nearly all of whose pages are absent: logits of 24 rows would take 1.6 GB."""
    cache = Cache([700, 37, 250, 0, 1, 64, 65, 333], 2, dim, fmt)
    table = torch.full((8, 2, 1 << 16), -1, dtype=torch.int32, device="cuda")
    table[:, :, :cache.table.shape[2]] = cache.table
    cache.table = table
    cache.paged = zc.PagedCache(cache.paged.k_pages, cache.paged.v_pages, table, cache.lengths, fmt, cache.ks, cache.vs)
    check(cache, [2, 1, 2, 0, 1, 2, 1, 1], 12, 200, 5, weights=True)


@pytest.mark.parametrize("q_lens,lens", [([1, 1], [9000, 40]), ([5, 1], [3000, 900]), ([300, 1], [700, 900])])
@pytest.mark.parametrize("weights", [False, True])
def test_scratch_of_the_callers(q_lens, lens, weights):
    """Of exactly the size that is asked for, whatever it holds before, and nothing behind it is touched."""
    cache = Cache(lens, 2, 128, E4M3)
    q, w = queries(sum(q_lens), 8, 128), [torch.zeros((2, 2, cache.paged.capacity), device="cuda") for _ in range(2)]
    more = dict(q_start=starts(q_lens), max_q_len=max(q_lens))
    want, want_lse = zc.attend(q, cache.paged, weights_out=w[0] if weights else None, **more)
    a = zc.AttendArgs()
    a.struct_size, a.n_tokens, a.n_q_heads, a.max_q_len, a.scale = C.sizeof(zc.AttendArgs), sum(q_lens), 8, max(q_lens), 128 ** -0.5
    a.d_q, a.d_q_start, a.d_out, a.d_lse = q.data_ptr(), more["q_start"].data_ptr(), want.data_ptr(), want_lse.data_ptr()
    a.q_token_stride = a.out_token_stride = 1024
    a.q_head_stride = a.out_head_stride = 128
    a.d_weights_out = w[0].data_ptr() if weights else None
    size = zc.lib().zc_attend_workspace_bytes(C.byref(a), None, cache.paged.ref)
    room = torch.full((size + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    out, lse = zc.attend(q, cache.paged, weights_out=w[1] if weights else None, ws=room[:size], **more)
    assert size and torch.equal(out, want) and torch.equal(lse, want_lse) and torch.equal(w[0], w[1])
    assert bool((room[size:] == 0xFF).all())
    if size > 16:
        with pytest.raises(zc.ZcError):
            zc.attend(q, cache.paged, weights_out=w[1] if weights else None, ws=room[:size - 1], **more)


@pytest.mark.parametrize("fmt", [BF16, E4M3])
def test_a_prompt_beside_long_decodes(fmt):
    check(Cache([300, 20011, 0, 5000, 1], 2, 64, fmt), [200, 1, 1, 3, 1], 4, weights=True)
    check(Cache([300, 20011, 0, 5000, 1], 2, 64, fmt), [200, 1, 1, 3, 1], 4, 9000, 20)
