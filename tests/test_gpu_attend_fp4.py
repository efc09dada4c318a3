"""Attention over pages of 4 bits (MXFP4, NVFP4) against its definition in 64 bits (tests/paged.py, where the tolerances are derived: MX weights are
rounded to BF16 as those of BF16 pages, NV weights to half precision as those of FP8 pages; the numbers of both formats go to the matrix
instructions exactly)."""
import pytest
import torch

from paper_2508_19263_amd import zc
from tests.paged import Cache, agree, attention, gen, starts
from tests.paged4 import MX, NV, Cache4
from tests.test_gpu_attend import check, queries

pytestmark = pytest.mark.gpu

FORMATS = [MX, NV]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 4, 7, 20])
def test_single_tokens(fmt, dim, group):
    check(Cache4([1, 0, 15, 16, 17, 31, 33, 1000, 2049], 2, dim, fmt), [1] * 9, group, single=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim,page", [(128, 16), (64, 16), (128, 32), (64, 64), (128, 1024)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (5, 3), (100, 70), (1000, 16)])
def test_windows_and_sinks(fmt, dim, page, window, sinks):
    check(Cache4([3001, 0, 64, 777, 1], 2, dim, fmt, page=page), [1, 1, 3, 5, 2], 3, window, sinks, weights=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_lens,lens", [([64, 1, 7], [64, 900, 20]), ([333, 0, 200], [333, 5, 641]), ([1025], [1500]), ([9, 40, 17], [3, 40, 0])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 5)])
def test_many_query_tokens(fmt, dim, q_lens, lens, window, sinks):
    check(Cache4(lens, 2, dim, fmt), q_lens, 4, window, sinks, weights=True)


@pytest.mark.parametrize("rows", [1, 16, 17, 32, 33, 64, 65, 128, 129])
@pytest.mark.parametrize("fmt", FORMATS)
def test_numbers_of_rows(rows, fmt):
    """Rows per K/V head on both sides of what a tile, a wavefront and a workgroup take, in one sequence, in many, over a prefix."""
    for window in (0, 200):
        check(Cache4([900], 2, 128, fmt), [rows], 1, window, 3, weights=True)
        check(Cache4([900], 2, 64, fmt), [1], rows, window, 3)
        check(Cache4([300, 200], 2, 128, fmt), [rows, 1], 1, window, 3, prefix=Cache4([333], 2, 128, fmt, seed=4))


@pytest.mark.parametrize("rows", [1, 17, 24, 25])
@pytest.mark.parametrize("fmt,dim", [(MX, 128), (NV, 64), (MX, 64), (NV, 128)])
def test_weights_of_numbers_of_rows(rows, fmt, dim):
    check(Cache4([700, 37, 2500], 3, dim, fmt), [rows, 1, max(1, rows - 1)], 1, 200, 5, weights=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_long_caches(fmt):
    check(Cache4([40007, 100, 12345], 1, 128, fmt), [1, 1, 1], 4, single=True, weights=True)
    check(Cache4([40007, 100, 12345], 1, 64, fmt), [1, 5, 3], 4, 30000, 100)
    check(Cache4([300, 8192, 0, 17001, 8193, 1, 8191] + [33 * i for i in range(10)], 16, 64, fmt), [1] * 17, 4, single=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("prefix,lens,q_lens", [(1, [1], [1]), (17, [0, 5, 40], [1, 1, 1]), (3000, [1, 100, 33, 257], [1, 1, 4, 2]), (5000, [20] * 40, [1] * 40),
                                                (257, [300, 10], [300, 3]), (0, [9, 4], [1, 1]), (100, [2, 0], [5, 3]), (40, [700, 20, 0, 5], [1, 9, 1, 4])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (64, 8)])
def test_shared_prefix(fmt, dim, prefix, lens, q_lens, window, sinks):
    check(Cache4(lens, 2, dim, fmt), q_lens, 4, window, sinks, prefix=Cache4([prefix], 2, dim, fmt, seed=9))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("scales", [False, True])
@pytest.mark.parametrize("scale", [0.0, -0.07, 1.5])
def test_scales(fmt, scales, scale):
    check(Cache4([300, 41], 2, 128, fmt, scales=scales), [1, 7], 4, scale=scale, weights=True)
    check(Cache4([300, 41], 2, 64, fmt, scales=scales), [1, 70], 4, scale=scale, weights=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("q_lens", [[1, 1], [100, 3]])
def test_absent_pages(fmt, q_lens):
    cache = Cache4([1000, 500], 2, 128, fmt)
    cache.table[0, :, 3:40] = -1
    cache.table[1, 0, 20] = cache.paged.n_pages
    cache.table[0, 1, 60] = 0x7FFFFFFF
    cache.table[1, 1, :] = -5                                    # nothing is left: empty rows
    check(cache, q_lens, 4, 300, 16, weights=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("name", ["k", "v"])
@pytest.mark.parametrize("q_len", [1, 3, 40, 200])
def test_what_is_not_finite_stays_with_those_who_see_it(fmt, dim, name, q_len):
    """Block scales that are NaN (and MX ones whose block is finite but for its largest numbers) in tokens that only the later queries see."""
    def edit(c):
        for i, t in enumerate((299, 298, 290, 250)):
            c.blocks[name][0, 0, t, i % c.blocks[name].shape[3]] = 255 if fmt == MX else 127 + 128 * (i & 1)
        c.blocks[name][0, 1, 150, -1] = 255 if fmt == MX else 127
    q, out, _ = check(Cache4([300], 2, dim, fmt, edit=edit), [q_len], 4, 60, 2)
    if q_len == 200:
        assert bool(out[:40].isfinite().all()) and not bool(out.isfinite().all())


@pytest.mark.parametrize("q_len", [1, 40, 200])
def test_largest_scales(q_len):
    """MX blocks whose scale is 2^126: the products of some of their elements are numbers, and those with 6 infinities."""
    def edit(c):
        c.blocks["v"][0, 0, 290, 1] = 253
        c.bits["v"][0, 0, 290, 16:32] = 0x01                     # one 0.5 in each pair
        c.bits["v"][0, 0, 290, 20] = 0x70                        # and a 6
        c.blocks["v"][0, 0, 280, 2] = 252
        c.bits["v"][0, 0, 280, 32:48] = 0x11
    cache = Cache4([300], 1, 128, MX, edit=edit)
    q = queries(q_len, 1, 128)
    out, _ = zc.attend(q, cache.paged, q_start=starts([q_len]), max_q_len=q_len)
    want, _, _, tol, _, _ = attention(q, [q_len], cache)
    seen = 290 - (300 - q_len)                                   # the first query that sees the infinity
    assert bool(out[max(seen, 0):, 0, 41].isinf().all()) and bool(out[:, 0, :32].isfinite().all())
    agree(out[..., :32], want[..., :32], tol[..., :32], "out")
    fine = want[:, 0, 32:41].abs() < 3e38
    assert bool(((out[:, 0, 32:41].to(torch.float64) - want[:, 0, 32:41]).abs()[fine] <= tol[:, 0, 32:41][fine]).all())


@pytest.mark.parametrize("fmt", FORMATS)
def test_scales_of_every_size(fmt):
    """Keys and values whose blocks' scales span what the format has, as far as results do not leave BF16's range."""
    def edit(c):
        g = gen(8)
        for name in "kv":
            b = c.blocks[name]
            if fmt == MX:                                        # keys to 2^-127, values from 2^-127 to 2^60
                b.copy_(torch.randint(0, 130 if name == "k" else 188, b.shape, generator=g, device="cuda").to(torch.uint8))
            else:
                b.copy_(torch.randint(0, 40 if name == "k" else 127, b.shape, generator=g, device="cuda").to(torch.uint8))
    check(Cache4([700, 33], 2, 128, fmt, edit=edit, scales=False), [1, 1], 4, weights=True)
    check(Cache4([700, 133], 2, 64, fmt, edit=edit, scales=False), [100, 33], 2, 70, 5, weights=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_page_numbers_whose_offsets_pass_32_bits(fmt):
    cache = Cache4([500, 37], 2, 128, fmt)
    n = (1 << 32) // 1024 + cache.paged.n_pages + 7
    pools = {}
    for name, x in cache.pools.items():
        pool = torch.empty((n,) + tuple(x.shape[1:]), dtype=x.dtype, device="cuda")
        pool[-x.shape[0]:] = x
        pool[:x.shape[0]] = 0x7F                                 # where offsets cut to 32 bits would read
        pools[name] = pool
    far = zc.PagedCache(pools["k"], pools["v"], (cache.table + (n - cache.paged.n_pages)).contiguous(), cache.lengths, fmt, cache.ks, cache.vs, pools["k_blocks"], pools["v_blocks"])
    for q, more in ((queries(2, 8, 128), {}), (queries(131, 8, 128), dict(q_start=starts([100, 31]), max_q_len=100))):
        want, want_lse = zc.attend(q, cache.paged, **more)
        got, lse = zc.attend(q, far, **more)
        assert torch.equal(got, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("fmt", FORMATS)
def test_the_same_call_gives_the_same_bits(fmt):
    cache = Cache4([9000, 4000], 2, 128, fmt)
    q = queries(2, 16, 128)
    w = [torch.zeros((2, 2, cache.paged.capacity), device="cuda") for _ in range(2)]
    a = zc.attend(q, cache.paged, weights_out=w[0])
    for _ in range(3):
        b = zc.attend(q, cache.paged, weights_out=w[1])
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(w[0], w[1])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page,into_page", [(16, 16), (32, 64)])
def test_eviction_moves_elements_and_block_scales(fmt, dim, page, into_page):
    cache = Cache4([400, 50, 0, 129], 2, dim, fmt, page=page)
    keep = 77
    into = Cache4([0] * 4, 2, dim, fmt, page=into_page, room=keep)
    w = torch.rand((4, 2, cache.paged.capacity), generator=gen(3), device="cuda")
    cache.table[0, 1, 1] = -1                                    # rows from an absent page are zero, block scales too
    kept = zc.evict(cache.paged, w, keep, into.paged, sinks=3, recent=20)
    assert into.lengths.tolist() == [77, 50, 0, 77]
    gone = set(range(page, 2 * page))
    for s in range(4):
        for h in range(2):
            n = min(cache.lens[s], keep)
            at, dst = kept[s, h, :n].to(torch.int64), torch.arange(n, device="cuda")
            for name in "kv":
                for kind, x in (("", cache.bits[name]), ("_blocks", cache.blocks[name])):
                    pool = into.pools[name + kind]
                    got = pool[into.table[s, h, dst // into_page].to(torch.int64), dst % into_page]
                    want = x[s, h, at].clone()
                    if (s, h) == (0, 1):
                        want[[i for i, t in enumerate(at.tolist()) if t in gone]] = 0
                    assert torch.equal(got, want)


def with_room(cache, tokens):
    """The cache with a table that has room for more tokens; the pages behind its own are absent."""
    seqs, heads, have = cache.table.shape
    more = torch.full((seqs, heads, -(-tokens // cache.page) - have), -1, dtype=torch.int32, device="cuda")
    cache.table = torch.cat([cache.table, more], dim=2).contiguous()
    p = cache.paged
    cache.paged = zc.PagedCache(p.k_pages, p.v_pages, cache.table, cache.lengths, p.fmt, p.k_scales, p.v_scales, p.k_blocks, p.v_blocks)
    return cache


@pytest.mark.parametrize("fmt,dim", [(MX, 128), (NV, 128), (MX, 64), (zc.FMT_BF16, 64), (zc.FMT_BF16, 128), (zc.FMT_FP8_E4M3, 64), (zc.FMT_FP8_E5M2, 128)])
@pytest.mark.parametrize("q_len", [1, 3, 8])
@pytest.mark.parametrize("weights", [False, True])
def test_room_for_more_than_the_caches_hold(fmt, dim, q_len, weights):
    """What may be read is more than 256 MB: these pages are loaded in another way (but for rows of less than 64 bytes)."""
    kind = Cache4 if fmt in (MX, NV) else Cache
    lens = [300, 1, 0, 1037, 64, 4099, 16, 17]
    cache = with_room(kind(lens, 8, dim, fmt), 40000)
    small = kind(lens, 8, dim, fmt)
    q_lens = [q_len] * len(lens)
    _, out, lse = check(cache, q_lens, 4, 0, 0, weights=weights)
    check(cache, q_lens, 4, 200, 5, weights=weights)             # (a window: less)
    want, want_lse = zc.attend(queries(len(lens) * q_len, 32, dim), small.paged, q_start=starts(q_lens), max_q_len=q_len)
    _, _, _, tol, tol_lse, _ = attention(queries(len(lens) * q_len, 32, dim), q_lens, small)
    agree(out, want.to(torch.float64), 2 * tol, "out")
    agree(lse, want_lse.to(torch.float64), 2 * tol_lse, "lse")


@pytest.mark.parametrize("fmt", FORMATS)
def test_rooms_and_longest_lengths(fmt):
    """Lengths past the room and past what the call was told is the longest, below zero: as with other formats."""
    cache = Cache4([100, 33, 64, 0], 2, 128, fmt)
    q = queries(4, 8, 128)
    want, want_lse = zc.attend(q, cache.paged)
    cache.lengths.copy_(torch.tensor([100, 33, 64, -7], dtype=torch.int32))
    got, lse = zc.attend(q, cache.paged)
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    full = Cache4([112, 112, 112, 112], 2, 128, fmt)
    want, want_lse = zc.attend(q, full.paged)
    full.lengths.fill_(2 ** 31 - 1)
    got, lse = zc.attend(q, full.paged)
    assert torch.equal(got, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_lens", [[1, 1], [40, 7], [300, 133]])
def test_negative_block_scales(dim, q_lens):
    """NV block scales are E4M3 numbers, and so may be negative (zc_kv_write gives none)."""
    def edit(c):
        for name in "kv":
            c.blocks[name] |= torch.randint(0, 2, c.blocks[name].shape, generator=gen(6), device="cuda").to(torch.uint8) << 7
    cache = Cache4([700, 133], 2, dim, NV, edit=edit)
    check(cache, q_lens, 4, weights=True)
    k, v = zc.read_kv(cache.paged, starts([700, 133]), 833)
    for s, first in ((0, 0), (1, 700)):
        for h in range(2):
            for name, got in (("k", k), ("v", v)):
                x = getattr(cache, name)[s, h, :cache.lens[s]].to(torch.float32) * getattr(cache, name + "s")[s, h]
                assert torch.equal(got[first:first + cache.lens[s], h], x.to(torch.bfloat16))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("length", [2559, 2560, 2561, 4095, 4096, 4097, 5120, 5121, 8191, 8192, 8193, 12288])
def test_where_long_caches_are_cut(fmt, length):
    check(Cache4([length, 5], 1, 128, fmt), [1, 1], 4, single=True)
    check(Cache4([length], 2, 64, fmt), [2], 3, length - 1, 1)


@pytest.mark.parametrize("fmt,dim", [(MX, 128), (NV, 128), (MX, 64), (NV, 64)])
@pytest.mark.parametrize("length", [255, 256, 257, 639, 641, 1024, 1025])
def test_short_caches(fmt, dim, length):
    """On both sides of the lengths between which a part has eight wavefronts; up to 16 rows and more."""
    cache = Cache4([length], 2, dim, fmt)
    check(cache, [1], 4, single=True)
    check(cache, [1], 16, length // 2, 5)
    check(cache, [3], 5)
    check(cache, [2], 9)
    cache.table[0, 1, ::3] = -1
    check(cache, [2], 7)


@pytest.mark.parametrize("fmt,dim", [(MX, 128), (NV, 64)])
@pytest.mark.parametrize("seqs,heads,length", [(8, 16, 1024), (43, 3, 1025), (8, 16, 1025), (16, 16, 2048), (16, 16, 2049), (257, 1, 700)])
def test_short_caches_of_many_heads(fmt, dim, seqs, heads, length):
    """128 and 256 (sequence, head)s, up to which longer caches are one part, and one more; lengths of all kinds and none."""
    lens = [length, 0, 1, 33, length - 1, 128] + [(i * 97) % (length if seqs < 99 else 60) for i in range(seqs - 6)]
    check(Cache4(lens, heads, dim, fmt), [1] * seqs, 4, single=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("seqs", [31, 32, 33])
def test_parts_of_many_heads(fmt, seqs):
    """512 (sequence, head)s, from which on parts are longer, one sequence less and one more; lengths of both kinds of parts and none."""
    lens = [0, 1, 2560, 2561, 4097, 5121, 6001] + [(i * 271) % 4000 for i in range(seqs - 7)]
    check(Cache4(lens, 16, 64, fmt), [1] * seqs, 4, single=True, weights=seqs != 32)


@pytest.mark.parametrize("fmt", FORMATS)
def test_on_another_stream_with_scratch_of_its_own_and_in_two_graphs(fmt):
    """Two graphs of one scratch, replayed in turn with the program's own work between them."""
    cache, prefix = Cache4([9000, 37, 500], 2, 128, fmt), Cache4([700], 2, 128, fmt, seed=3)
    q, big = queries(3, 8, 128), queries(211, 8, 128, 9)
    many = dict(q_start=starts([200, 1, 10]), max_q_len=200)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(q), torch.zeros_like(big), torch.zeros_like(q)]
    calls = [lambda o, **m: zc.attend(q, cache.paged, out=o, **m), lambda o, **m: zc.attend(big, cache.paged, out=o, **many, **m),
             lambda o, **m: zc.attend_shared(q, prefix.paged, cache.paged, out=o, **m)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for call, o in zip(calls, outs):
            call(o, ws=ws)
    side.synchronize()
    want = [torch.zeros_like(o) for o in outs]
    for call, o in zip(calls, want):
        call(o)
    for o, w in zip(outs, want):
        assert torch.equal(o, w)
    graphs = []
    for call, o in zip(calls, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(o, ws=ws)
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=gen(i), device="cuda"))
        big.copy_(torch.randn(big.shape, generator=gen(i + 9), device="cuda"))
        for graph in graphs:
            graph.replay()
        if i % 2:
            torch.cuda.synchronize()
        for call, o, w in zip(calls, outs, want):
            call(w)
            assert torch.equal(o, w)
