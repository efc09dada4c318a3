"""Attention over K/V pages against its definition in 64 bits (tests/paged.py, where the tolerances are derived)."""
import math

import pytest
import torch

from paper_2508_19263_amd import zc
from tests.paged import JUNK, STORE, Cache, agree, attention, gen, starts, stored

pytestmark = pytest.mark.gpu

BF16, E4M3, E5M2 = zc.FMT_BF16, zc.FMT_FP8_E4M3, zc.FMT_FP8_E5M2


def queries(n, heads, dim, seed=5):
    return torch.randn((n, heads, dim), generator=gen(seed), device="cuda").to(torch.bfloat16)


def check(cache, q_lens, group, window=0, sinks=0, prefix=None, weights=False, single=False, seed=5, **more):
    heads, dim = cache.k.shape[1], cache.k.shape[3]
    q = queries(sum(q_lens), heads * group, dim, seed)
    if not single:
        more.update(q_start=starts(q_lens), max_q_len=max(q_lens + [1]))
    w = torch.rand((len(q_lens), heads, cache.paged.capacity), generator=gen(seed + 1), device="cuda") if weights else None
    if prefix is not None:
        out, lse = zc.attend_shared(q, prefix.paged, cache.paged, window=window, sinks=sinks, **more)
    elif weights:
        w_out = torch.full_like(w, -7.0)
        out, lse = zc.attend(q, cache.paged, window=window, sinks=sinks, weights=w, weights_out=w_out, **more)
    else:
        out, lse = zc.attend(q, cache.paged, window=window, sinks=sinks, **more)
    torch.cuda.synchronize()
    want, want_lse, want_w, tol, tol_lse, tol_w = attention(q, q_lens, cache, prefix, window, sinks, more.get("scale"), w)
    agree(out, want, tol, "out")
    agree(lse, want_lse, tol_lse, "lse")
    if weights:
        for s, n in enumerate(cache.lens):
            agree(w_out[s, :, :n], want_w[s, :, :n], tol_w[s, :, :n], "weights")
            assert bool((w_out[s, :, n:] == -7.0).all())
    return q, out, lse


@pytest.mark.parametrize("fmt", [BF16, E4M3, E5M2])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 4, 7, 20])
def test_single_tokens(fmt, dim, group):
    check(Cache([1, 0, 15, 16, 17, 31, 33, 1000, 2049], 2, dim, fmt), [1] * 9, group, single=True)


@pytest.mark.parametrize("fmt", [BF16, E4M3, E5M2])
@pytest.mark.parametrize("page", [16, 32, 64, 1024])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (5, 3), (100, 4), (100, 70), (1000, 16), (5000, 9)])
def test_windows_and_sinks(fmt, page, window, sinks):
    check(Cache([3001, 0, 64, 777, 1], 2, 128, fmt, page=page), [1, 1, 3, 5, 2], 3, window, sinks, weights=True)


@pytest.mark.parametrize("fmt", [BF16, E4M3, E5M2])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_lens,lens", [([64, 1, 7], [64, 900, 20]), ([333, 0, 200], [333, 5, 641]), ([1025], [1500]), ([9, 40, 17], [3, 40, 0])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 5), (257, 0)])
def test_many_query_tokens(fmt, dim, q_lens, lens, window, sinks):
    """Prompts whole and in pieces; the last case has more query tokens than cached ones: the first of them see nothing."""
    check(Cache(lens, 2, dim, fmt), q_lens, 4, window, sinks, weights=True)


@pytest.mark.parametrize("rows", [1, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 127, 128, 129])
@pytest.mark.parametrize("window", [0, 200])
def test_numbers_of_rows(rows, window):
    """Rows per K/V head on both sides of what a tile, a wavefront and a workgroup take, in one sequence, in many, over a prefix."""
    for fmt in (BF16, E4M3):
        check(Cache([900], 2, 128, fmt), [rows], 1, window, 3, weights=True)
        check(Cache([900], 2, 64, fmt), [1], rows, window, 3)
        check(Cache([40 + i for i in range(rows)], 2, 64, fmt), [1] * rows, 1, window, 3, prefix=Cache([700], 2, 64, fmt, seed=4))
        check(Cache([300, 200], 2, 128, fmt), [rows, 1], 1, window, 3, prefix=Cache([333], 2, 128, fmt, seed=4))


@pytest.mark.parametrize("rows", [1, 15, 16, 17, 23, 24, 25, 33])
@pytest.mark.parametrize("fmt,dim", [(BF16, 128), (E4M3, 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 5)])
def test_weights_of_numbers_of_rows(rows, fmt, dim, window, sinks):
    check(Cache([700, 37, 2500], 3, dim, fmt), [rows, 1, max(1, rows - 1)], 1, window, sinks, weights=True)
    if rows % 4 == 0:
        check(Cache([700, 37, 2500], 3, dim, fmt), [4, 0, 3], rows // 4, window, sinks, weights=True)


@pytest.mark.parametrize("fmt", [BF16, E4M3])
@pytest.mark.parametrize("group,heads", [(1, 1), (2, 5), (8, 1), (64, 1)])
def test_head_layouts(fmt, group, heads):
    check(Cache([700, 33], heads, 128, fmt), [20, 1], group, 300, 4, weights=True)


@pytest.mark.parametrize("fmt", [BF16, E4M3, E5M2])
def test_long_cache(fmt):
    check(Cache([40007, 100, 12345], 1, 128, fmt), [1, 1, 1], 4, single=True, weights=True)
    check(Cache([40007, 100, 12345], 1, 64, fmt), [1, 5, 3], 4, 30000, 100)


@pytest.mark.parametrize("fmt", [BF16, E4M3])
@pytest.mark.parametrize("group,window,weights", [(1, 0, False), (4, 9000, True), (20, 0, False)])
def test_one_long_cache_among_short_ones(fmt, group, window, weights):
    # more (sequence, head) pairs than compute units, and parts that only the long cache fills
    lens = [300, 8192, 0, 17001, 8193, 1, 8191] + [33 * i for i in range(10)]
    check(Cache(lens, 16, 64, fmt), [1] * 17, group, window, 4 if window else 0, weights=weights, single=True)


@pytest.mark.parametrize("fmt", [BF16, E4M3, E5M2])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("prefix,lens,q_lens", [(1, [1], [1]), (17, [0, 5, 40], [1, 1, 1]), (3000, [1, 100, 33, 257], [1, 1, 4, 2]), (5000, [20] * 40, [1] * 40),
                                                (257, [300, 10], [300, 3]), (0, [9, 4], [1, 1]), (100, [2, 0], [5, 3]),
                                                (3000, [30] * 10, [1] * 10), (900, [64, 70], [15, 9]), (40, [700, 20, 0, 5], [1, 9, 1, 4])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (64, 8), (2000, 130)])
def test_shared_prefix(fmt, dim, prefix, lens, q_lens, window, sinks):
    """A query whose sequence has fewer tokens of its own than it has queries is positioned in the prefix."""
    pre = Cache([prefix], 2, dim, fmt, seed=9)
    check(Cache(lens, 2, dim, fmt), q_lens, 4, window, sinks, prefix=pre)


def test_shared_prefix_with_sinks_that_reach_into_the_sequences():
    check(Cache([500, 90], 2, 128, E4M3), [2, 1], 4, 20, 150, prefix=Cache([100], 2, 128, E4M3, page=32, seed=9))


@pytest.mark.parametrize("scale", [0.0, -0.07, 1.5])
def test_scales_of_logits(scale):
    check(Cache([300, 41], 2, 128, E4M3), [1, 7], 4, scale=scale, weights=True)
    check(Cache([300, 41], 2, 128, BF16, scales=True), [1, 70], 4, scale=scale, weights=True)


@pytest.mark.parametrize("q_lens", [[1, 1], [100, 3]])
def test_absent_pages(q_lens):
    """Pages that the window has left behind are given back: their numbers are nobody's.  An absent page inside the window hides its tokens."""
    cache = Cache([1000, 500], 2, 128, E4M3)
    cache.table[0, :, 3:40] = -1
    cache.table[1, 0, 20] = cache.paged.n_pages
    cache.table[0, 1, 60] = 0x7FFFFFFF
    cache.table[1, 1, :] = -5                                    # nothing is left: empty rows
    check(cache, q_lens, 4, 300, 16, weights=True)


@pytest.mark.parametrize("fmt", [BF16, E4M3, E5M2])
@pytest.mark.parametrize("name", ["k", "v"])
@pytest.mark.parametrize("q_len", [1, 3, 40, 200])
def test_what_is_not_finite_stays_with_those_who_see_it(fmt, name, q_len):
    """NaN and infinities in tokens that only the later queries see: the earlier ones are as if they were not there."""
    def edit(c):
        x = getattr(c, name)
        wild = {BF16: [0x7F80, -128, 0x7FC0], E4M3: [0x7F, 0xFF], E5M2: [0x7C, 0xFC, 0x7F]}[fmt]   # -128: 0xFF80
        for i, t in enumerate((299, 298, 290, 250)):
            x[0, 0, t, 5 + 9 * i] = wild[i % len(wild)]
        x[0, 1, 150, 64] = wild[0]
    q, out, _ = check(Cache([300], 2, 128, fmt, edit=edit), [q_len], 4, 60, 2)
    if q_len == 200:
        assert bool(out[:40].isfinite().all()) and not bool(out.isfinite().all())


@pytest.mark.parametrize("fmt", [BF16, E4M3])
@pytest.mark.parametrize("q_len,before", [(3, 0), (100, 0), (2, 3000), (100, 3000)])
def test_a_query_that_is_not_a_number(fmt, q_len, before):
    """It is the business of its own row, and of the weights of what it sees; also where a cache is split."""
    cache = Cache([300, 200 + before], 1, 128, fmt)
    if before:
        q = queries(2 * q_len, 4, 128)
        q[q_len:, 2] = float("nan")
        out, lse = zc.attend(q, cache.paged, q_start=starts([q_len, q_len]), max_q_len=q_len)
        shared, shared_lse = zc.attend_shared(q, Cache([3000], 1, 128, fmt, seed=3).paged, cache.paged, q_start=starts([q_len, q_len]), max_q_len=q_len)
        for o, z in ((out, lse), (shared, shared_lse)):
            assert bool(o[q_len:, 2].isnan().all()) and bool(z[q_len:, 2].isnan().all())
            assert int(o.isnan().any(dim=2).sum()) == q_len and int(z.isfinite().sum()) == z.numel() - q_len
        return
    q = queries(q_len + 1, 4, 128)
    bad = q_len - 2                                              # the last but one of the first sequence
    q[bad, 1, 7] = float("nan")
    w_out = torch.zeros((2, 1, cache.paged.capacity), device="cuda")
    out, lse = zc.attend(q, cache.paged, q_start=starts([q_len, 1]), max_q_len=q_len, window=50, sinks=3, weights_out=w_out)
    want, want_lse, want_w, tol, tol_lse, tol_w = attention(q, [q_len, 1], cache, None, 50, 3, None, torch.zeros_like(w_out))
    agree(out, want, tol.nan_to_num(0), "out")
    agree(lse, want_lse, tol_lse.nan_to_num(0), "lse")
    for s, n in enumerate(cache.lens):
        agree(w_out[s, :, :n], want_w[s, :, :n], tol_w[s, :, :n].nan_to_num(0), "weights")
    assert bool(out[bad, 1].isnan().all()) and int(out.isnan().any(dim=2).sum()) == 1
    assert bool(w_out[0, 0, 299].isfinite()) and bool(w_out[0, 0, 298].isnan()) and bool(w_out[0, 0, 100].isfinite())


def test_strided_queries_and_results():
    cache = Cache([200, 50, 17], 2, 128, E4M3)
    q_lens = [3, 1, 40]
    wide = torch.randn((44, 12, 384), generator=gen(3), device="cuda").to(torch.bfloat16)
    q, room = wide[:, 1:9, 128:256], torch.zeros((44, 16, 136), dtype=torch.bfloat16, device="cuda")
    out = room[:, ::2, :128]
    zc.attend(q, cache.paged, q_start=starts(q_lens), max_q_len=40, out=out)
    want, _, _, tol, _, _ = attention(q, q_lens, cache)
    agree(out, want, tol, "out")
    assert not bool(room[:, 1::2].any()) and not bool(room[:, :, 128:].any())


def test_query_tokens_of_no_sequence_are_left_alone():
    cache = Cache([100, 200], 1, 64, E4M3)
    q = queries(9, 4, 64)
    start = torch.tensor([2, 4, 5], dtype=torch.int32, device="cuda")          # tokens 0, 1 and 5 .. 8 are nobody's
    for shared in (False, True):
        out, lse = torch.full_like(q, 3.0), torch.full((9, 4), 3.0, device="cuda")
        pre = Cache([300], 1, 64, E4M3, seed=4)
        if shared:
            zc.attend_shared(q, pre.paged, cache.paged, q_start=start, max_q_len=2, out=out, lse=lse)
        else:
            zc.attend(q, cache.paged, q_start=start, max_q_len=2, out=out, lse=lse)
        want, want_lse, _, tol, tol_lse, _ = attention(q[2:5], [2, 1], cache, pre if shared else None)
        agree(out[2:5], want, tol, "out")
        agree(lse[2:5], want_lse, tol_lse, "lse")
        assert bool((out[:2] == 3).all()) and bool((out[5:] == 3).all()) and bool((lse[:2] == 3).all()) and bool((lse[5:] == 3).all())


def test_lengths_beyond_the_room_and_below_zero():
    cache = Cache([64, 30], 1, 64, E4M3)
    q = queries(2, 4, 64)
    want, _ = zc.attend(q, cache.paged)
    cache.lengths[0] = 1000                                      # 64 tokens is what the table has room for
    got, _ = zc.attend(q, cache.paged)
    assert torch.equal(got, want)
    cache.lengths[0], cache.lengths[1] = 64, -3
    got, lse = zc.attend(q, cache.paged, max_kv_len=64)
    assert torch.equal(got[0], want[0]) and not bool(got[1].any()) and bool((lse[1] == -math.inf).all())


@pytest.mark.parametrize("fmt", [BF16, E4M3])
def test_page_numbers_whose_offsets_pass_32_bits(fmt):
    cache = Cache([500, 37], 2, 128, fmt)
    kp, vp = cache.paged.k_pages, cache.paged.v_pages
    page_bytes = kp[0].numel() * kp.element_size()
    n = (1 << 32) // page_bytes + kp.shape[0] + 7
    pools = []
    for x in (kp, vp):
        pool = torch.empty((n,) + tuple(x.shape[1:]), dtype=x.dtype, device="cuda")
        pool[-x.shape[0]:] = x
        pool[:x.shape[0]] = JUNK[fmt]                            # where offsets cut to 32 bits would read
        pools.append(pool)
    q = queries(2, 8, 128)
    want, want_lse = zc.attend(q, cache.paged)
    far = zc.PagedCache(pools[0], pools[1], (cache.table + (n - kp.shape[0])).contiguous(), cache.lengths, fmt, cache.ks, cache.vs)
    got, lse = zc.attend(q, far)
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    into = Cache([0, 0], 2, 128, fmt, room=100)
    w = torch.rand((2, 2, far.capacity), generator=gen(2), device="cuda")
    near = zc.evict(cache.paged, w, 90, into.paged)
    k_near = into.paged.k_pages.clone()
    kept = zc.evict(far, w, 90, into.paged)
    assert torch.equal(kept, near) and torch.equal(into.paged.k_pages, k_near)


def test_the_same_call_gives_the_same_bits():
    cache = Cache([9000, 4000], 2, 128, BF16)
    q = queries(2, 16, 128)
    w = [torch.zeros((2, 2, cache.paged.capacity), device="cuda") for _ in range(2)]
    a = zc.attend(q, cache.paged, weights_out=w[0])
    for _ in range(3):
        b = zc.attend(q, cache.paged, weights_out=w[1])
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(w[0], w[1])


def test_weights_in_place():
    cache = Cache([900, 400], 2, 128, E4M3)
    q = queries(2, 16, 128)
    w = torch.rand((2, 2, cache.paged.capacity), generator=gen(2), device="cuda")
    apart = torch.zeros_like(w)
    zc.attend(q, cache.paged, weights=w, weights_out=apart)
    zc.attend(q, cache.paged, weights=w, weights_out=w)
    assert torch.equal(w[0, :, :900], apart[0, :, :900]) and torch.equal(w[1, :, :400], apart[1, :, :400])


def test_on_another_stream_and_in_a_graph():
    cache, pre = Cache([3000, 700, 1], 2, 128, E4M3), Cache([2000], 2, 128, E4M3, seed=8)
    q = queries(3, 8, 128)
    w = torch.zeros((3, 2, cache.paged.capacity), device="cuda")
    want, want_lse = zc.attend(q, cache.paged, weights_out=w)
    shared, _ = zc.attend_shared(q, pre.paged, cache.paged)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got, lse = zc.attend(q, cache.paged)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    w2 = torch.zeros_like(w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, lse = zc.attend(q, cache.paged, weights_out=w2)
        got_shared, _ = zc.attend_shared(q, pre.paged, cache.paged)
    for i in range(4):
        got.zero_()
        got_shared.zero_()
        w2.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.randn((1000, 1000), device="cuda").sum()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(got_shared, shared) and torch.equal(w2, w)
    cache.lengths[0] = 1234                                      # lengths are read when the graph runs
    want, _ = zc.attend(q, cache.paged)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_pages_of_a_container():
    """What the codec decodes is what attention reads: a cache compressed in pages and decoded again gives the same result."""
    cache = Cache([512, 512], 2, 128, E4M3)
    q = queries(2, 8, 128)
    want, _ = zc.attend(q, cache.paged)
    p = zc.params(zc.FMT_FP8_E4M3, 2048, streams=8)
    pools = []
    for x in (cache.paged.k_pages, cache.paged.v_pages):
        comp, info = zc.compress(x, x.numel(), p)
        pools.append(zc.decompress(comp, info)[0].view(x.shape))
    got, _ = zc.attend(q, zc.PagedCache(pools[0], pools[1], cache.table, cache.lengths, E4M3, cache.ks, cache.vs))
    assert torch.equal(got, want)


def test_no_query_tokens():
    cache = Cache([40, 9], 1, 64, BF16)
    w = torch.rand((2, 1, cache.paged.capacity), generator=gen(2), device="cuda")
    w_out = torch.zeros_like(w)
    out, _ = zc.attend(queries(0, 4, 64), cache.paged, q_start=starts([0, 0]), weights=w, weights_out=w_out)
    assert out.shape == (0, 4, 64) and torch.equal(w_out[0, 0, :40], w[0, 0, :40]) and torch.equal(w_out[1, 0, :9], w[1, 0, :9])
