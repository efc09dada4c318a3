"""Rows written to and read from K/V pages: stored bits are those of the definition (tests/paged4.py), everything else is as it was."""
import pytest
import torch

from paper_2508_19263_amd import workloads as wl
from paper_2508_19263_amd import zc
from tests.paged import gen, starts
from tests.paged4 import BLOCK, E4M3, E5M2, MX, NV, element_value, nearest, quantised4, scale_value

pytestmark = pytest.mark.gpu

BF16, F8, F8B = zc.FMT_BF16, zc.FMT_FP8_E4M3, zc.FMT_FP8_E5M2
FORMATS = [BF16, F8, F8B, MX, NV]


def quantised(y, fmt):
    """float32 [..., dim] -> (stored elements, block scales or None)."""
    if fmt == BF16:
        return y.to(torch.bfloat16).view(torch.int16), None
    if fmt in BLOCK:
        return quantised4(y, fmt)
    code = nearest(y.to(torch.float64).nan_to_num(0.0), E4M3 if fmt == F8 else E5M2)
    code = torch.where(y.isnan(), torch.full_like(code, 0x7F), code) | torch.signbit(y).to(torch.int64) << 7
    return code.to(torch.uint8), None


def numbers(bits, blocks, fmt, scale):
    """Stored elements (and block scales) times the scale, in 32 bits, as BF16."""
    if fmt == BF16:
        x = bits.view(torch.bfloat16).to(torch.float32)
        if scale is None:
            return x.to(torch.bfloat16)
    elif fmt in BLOCK:
        x = (element_value(bits).unflatten(-1, (-1, BLOCK[fmt])) * scale_value(blocks, fmt).unsqueeze(-1)).flatten(-2).to(torch.float32)
    else:
        x = bits.view(torch.float8_e4m3fn if fmt == F8 else torch.float8_e5m2).to(torch.float32)
    return (x if scale is None else x * scale).to(torch.bfloat16)


def the_same(got, want, what):
    """Bit for bit, but that a NaN is a NaN."""
    a, b = got.isnan() if got.is_floating_point() else None, want.isnan() if want.is_floating_point() else None
    if a is not None:
        assert torch.equal(a, b), what
        got, want = torch.where(a, torch.zeros_like(got), got).view(torch.int16), torch.where(b, torch.zeros_like(want), want).view(torch.int16)
    assert torch.equal(got, want), "%s: %d of %d differ" % (what, int((got != want).sum()), got.numel())


class Pages:
    """An empty cache: pools of random bits (what was there before), a table in random order."""

    def __init__(self, lens, heads, dim, fmt, page=16, scales=False, seed=2, table=None, n_pages=None):
        g = gen(seed)
        per = max(1, -(-max(lens) // page))
        used = len(lens) * heads * per
        n = n_pages or used + 3
        width = {BF16: dim, F8: dim, F8B: dim}.get(fmt, dim // 2)
        self.fmt, self.lens, self.heads, self.dim, self.page = fmt, list(lens), heads, dim, page
        self.pools = {}
        for name in "kv":
            x = torch.randint(0, 256, (n, page, width * (2 if fmt == BF16 else 1)), generator=g, device="cuda").to(torch.uint8)
            self.pools[name] = x.view(torch.int16) if fmt == BF16 else x
            if fmt in BLOCK:
                self.pools[name + "_blocks"] = torch.randint(0, 256, (n, page, dim // BLOCK[fmt]), generator=g, device="cuda").to(torch.uint8)
        self.table = (torch.randperm(n, generator=g, device="cuda")[:used].view(len(lens), heads, per).to(torch.int32) if table is None else table)
        self.lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.scales = {name: torch.rand((len(lens), heads), generator=g, device="cuda") + 0.01 if scales else None for name in "kv"}
        self.paged = zc.PagedCache(self.pools["k"], self.pools["v"], self.table, self.lengths, fmt, self.scales["k"], self.scales["v"],
                                   self.pools.get("k_blocks"), self.pools.get("v_blocks"))

    def places(self, q_lens, first=0):
        """(token, seq, position) of every token that has one in a page."""
        t = first
        for s, n in enumerate(q_lens):
            for i in range(n):
                yield t, s, self.lens[s] - n + i
                t += 1


def expected(pages, k, v, q_lens, first=0):
    """The pools after the write."""
    pools = {name: x.clone() for name, x in pages.pools.items()}
    capacity = pages.table.shape[2] * pages.page
    for name, x in (("k", k), ("v", v)):
        for t, s, at in pages.places(q_lens, first):
            if not 0 <= at < capacity:
                continue
            y = x[t].to(torch.float32)
            if pages.scales[name] is not None:
                scale = pages.scales[name][s].unsqueeze(1)
                most = torch.finfo(torch.float32).max
                y = torch.where(scale == 0, torch.zeros_like(y), y * (1.0 / scale).clamp(-most, most))
            bits, blocks = quantised(y, pages.fmt)
            if pages.fmt == BF16 and pages.scales[name] is None:
                bits = x[t].view(torch.int16)
            for h in range(pages.heads):
                page = int(pages.table[s, h, at // pages.page])
                if 0 <= page < pools[name].shape[0]:
                    pools[name][page, at % pages.page] = bits[h]
                    if blocks is not None:
                        pools[name + "_blocks"][page, at % pages.page] = blocks[h]
    return pools


def compare(pages, pools):
    for name, want in pools.items():
        got = pages.pools[name]
        if pages.fmt == BF16:
            got, want = got.view(torch.bfloat16), want.view(torch.bfloat16)
        if pages.fmt in (F8, F8B) or name.endswith("blocks"):
            kind = {F8: torch.float8_e4m3fn, F8B: torch.float8_e5m2}.get(pages.fmt)
            if kind is None and pages.fmt == NV:
                kind = torch.float8_e4m3fn
            if kind is not None:                                 # any NaN
                a, b = got.view(kind).to(torch.float32).isnan(), want.view(kind).to(torch.float32).isnan()
                assert torch.equal(a, b), name
                got, want = torch.where(a, torch.zeros_like(got), got), torch.where(b, torch.zeros_like(want), want)
        the_same(got, want, name)


def rows(n, heads, dim, seed=7, wide=False):
    g = gen(seed)
    if wide:                                                     # heads of a fused projection, every other token
        x = torch.randn((n * 2, heads * 3 + 1, dim + 8), generator=g, device="cuda").to(torch.bfloat16)
        k, v = x[::2, 1:heads + 1, :dim], x[1::2, heads:2 * heads, 8:]
    else:
        k, v = (torch.randn((n, heads, dim), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    size = torch.exp2(torch.randint(-12, 9, (n, heads, 1), generator=g, device="cuda").to(torch.float32)).to(torch.bfloat16)
    k.mul_(size)
    v[: n // 2].mul_(size[: n // 2])
    return k, v


def write_and_check(pages, q_lens, single=False, wide=False, k=None, v=None):
    if k is None:
        k, v = rows(sum(q_lens), pages.heads, pages.dim, wide=wide)
    want = expected(pages, k, v, q_lens)
    zc.write_kv(k, v, pages.paged, None if single else starts(q_lens))
    torch.cuda.synchronize()
    compare(pages, want)
    return k, v


def read_and_check(pages, q_lens, single=False):
    got = zc.read_kv(pages.paged, None if single else starts(q_lens), sum(q_lens))
    torch.cuda.synchronize()
    capacity = pages.table.shape[2] * pages.page
    for name, x in zip("kv", got):
        want = torch.zeros_like(x)
        for t, s, at in pages.places(q_lens):
            for h in range(pages.heads):
                page = int(pages.table[s, h, at // pages.page]) if 0 <= at < capacity else -1
                if 0 <= page < pages.pools[name].shape[0]:
                    blocks = pages.pools.get(name + "_blocks")
                    want[t, h] = numbers(pages.pools[name][page, at % pages.page], None if blocks is None else blocks[page, at % pages.page], pages.fmt,
                                         None if pages.scales[name] is None else pages.scales[name][s, h])
        the_same(x, want, name)
    return got


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scales", [False, True])
def test_a_token_of_each_sequence(fmt, dim, scales):
    pages = Pages([1, 16, 17, 33, 5, 100], 3, dim, fmt, scales=scales)
    write_and_check(pages, [1] * 6, single=True)
    read_and_check(pages, [1] * 6, single=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim,page,heads", [(128, 16, 2), (64, 16, 5), (128, 64, 1), (64, 1024, 2)])
@pytest.mark.parametrize("q_lens", [[1], [3, 0, 16, 1], [33, 17], [5, 0, 0, 70], [0, 0]])
def test_several_tokens(fmt, dim, page, heads, q_lens):
    """Pages that begin and end inside what is written; sequences without tokens."""
    pages = Pages([n + 7 * i for i, n in enumerate(q_lens)], heads, dim, fmt, page=page, scales=fmt != BF16 and page == 16)
    write_and_check(pages, q_lens, wide=True)
    read_and_check(pages, q_lens)


@pytest.mark.parametrize("fmt", FORMATS)
def test_what_has_no_place_is_left_out(fmt):
    """Positions below zero (more tokens than the length) and past the table's room, absent pages."""
    pages = Pages([3, 48, 20, 10], 2, 128, fmt)
    pages.lengths[1], pages.lens[1] = 51, 51                     # the table has room for 48
    pages.lengths[3], pages.lens[3] = -4, 0
    pages.table[2, 0, 0], pages.table[2, 1, 1] = -1, pages.paged.n_pages
    write_and_check(pages, [5, 7, 18, 2])
    read_and_check(pages, [5, 7, 18, 2])


@pytest.mark.parametrize("fmt", FORMATS)
def test_tokens_of_no_sequence(fmt):
    pages = Pages([20, 30], 1, 64, fmt)
    k, v = rows(9, 1, 64)
    start = torch.tensor([2, 4, 5], dtype=torch.int32, device="cuda")
    want = expected(pages, k, v, [2, 1], first=2)
    zc.write_kv(k, v, pages.paged, start)
    compare(pages, want)
    whole = zc.read_kv(pages.paged, starts([2, 1]), 3)
    out = torch.full((9, 1, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    k2, _ = zc.read_kv(pages.paged, start, k=out)
    assert k2 is out and bool((out[:2] == 3).all()) and bool((out[5:] == 3).all())
    the_same(out[2:5], whole[0], "k")


@pytest.mark.parametrize("fmt", FORMATS)
def test_numbers_of_every_kind(fmt):
    """All BF16 numbers, NaN and infinities among them: a block, or an element, that holds a NaN is one, an infinity is the largest number."""
    every = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16).view(torch.bfloat16)
    order = torch.randperm(65536, generator=gen(4), device="cuda")
    for x in (every, every[order], torch.where(every.isfinite(), every, torch.zeros_like(every))[order]):
        k, v = x.view(64, 8, 128), x.flip(0).view(64, 8, 128)
        pages = Pages([64], 8, 128, fmt)
        write_and_check(pages, [64], k=k, v=v)
        read_and_check(pages, [64])


@pytest.mark.parametrize("fmt", FORMATS)
def test_ties_and_scales(fmt):
    """Numbers half way between neighbours, and scales of sequences and heads that are large, small, negative, zero, and not numbers."""
    base = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0], device="cuda")
    x = (base.repeat(8) * torch.exp2(torch.arange(-30, 34, device="cuda")).view(-1, 1)).view(64, 1, 128).expand(-1, 2, -1)
    k, v = x.to(torch.bfloat16).contiguous(), (x * 1.125).to(torch.bfloat16).contiguous()
    write_and_check(Pages([64], 2, 128, fmt), [64], k=k, v=v)
    pages = Pages([64] * 4, 2, 128, fmt, scales=True)
    for name in "kv":
        pages.scales[name].copy_(torch.tensor([[1.0, 2.0 ** -40], [3.0e5, -0.7], [0.0, float("nan")], [float("inf"), 1e-30]], device="cuda"))
    write_and_check(pages, [64] * 4, k=k.repeat(4, 1, 1), v=v.repeat(4, 1, 1))
    read_and_check(pages, [64] * 4)


@pytest.mark.parametrize("fmt", [MX, NV])
def test_what_the_library_calls_these_formats(fmt):
    """MXFP4 as written is what the generators of compressed weights give (NVFP4 with their scale of the whole tensor)."""
    pages = Pages([256], 4, 128, fmt, scales=fmt == NV)
    k, v = rows(256, 4, 128)
    k, v = k.clamp(-60, 60), v.clamp(-60, 60)
    if fmt == NV:
        for name, x in (("k", k), ("v", v)):
            pages.scales[name].fill_(float((x.to(torch.float32).reshape(-1, 16).abs().amax(dim=1) / 6.0).max() / 448.0))
    zc.write_kv(k, v, pages.paged, starts([256]))
    if fmt == MX:
        for name, x in (("k", k), ("v", v)):
            bits, blocks = wl.mxfp4_bits(x.to(torch.float32))
            got = pages.pools[name][pages.table[0].to(torch.int64)].view(4, 256, 64).transpose(0, 1)
            assert torch.equal(got.reshape(-1), bits.reshape(-1))
            assert torch.equal(pages.pools[name + "_blocks"][pages.table[0].to(torch.int64)].view(4, 256, 4).transpose(0, 1).reshape(-1), blocks)
    else:
        for name, x in (("k", k), ("v", v)):                     # (y = x / S is rounded before the block's scale is taken: a step of it, in a few blocks)
            _, blocks = wl.nvfp4_bits(x.to(torch.float32))
            got = pages.pools[name + "_blocks"][pages.table[0].to(torch.int64)].view(4, 256, 8).transpose(0, 1).reshape(-1)
            off = (got.to(torch.int32) - blocks.to(torch.int32)).abs()
            assert int(off.max()) <= 1 and int((off > 0).sum()) <= 8


@pytest.mark.parametrize("n_seqs", [63, 64, 65, 130, 1024, 1025, 3000])
def test_many_sequences(n_seqs):
    """On both sides of how sequences are found."""
    q_lens = [(i * 7) % 4 for i in range(n_seqs)]
    pages = Pages([16] * n_seqs, 1, 64, F8)
    n = sum(q_lens)
    k, v = rows(n, 1, 64)
    zc.write_kv(k, v, pages.paged, starts(q_lens))
    got_k, got_v = zc.read_kv(pages.paged, starts(q_lens), n)
    for x, got in ((k, got_k), (v, got_v)):
        bits, _ = quantised(x.to(torch.float32), F8)
        the_same(got, numbers(bits, None, F8, None), "rows")
    seq = torch.repeat_interleave(torch.arange(n_seqs, device="cuda"), torch.tensor(q_lens, device="cuda"))
    at = 16 - torch.tensor(q_lens, device="cuda")[seq] + torch.arange(n, device="cuda") - starts(q_lens).to(torch.int64)[seq]
    bits, _ = quantised(k.to(torch.float32), F8)
    assert torch.equal(pages.pools["k"][pages.table[seq, 0, 0].to(torch.int64), at], bits[:, 0])


@pytest.mark.parametrize("fmt", [F8, MX])
def test_page_numbers_whose_offsets_pass_32_bits(fmt):
    page_bytes = 16 * 128 // (1 if fmt == F8 else 2)
    n = (1 << 32) // page_bytes + 50
    table = torch.tensor([[[n - 1, 3], [n - 40, n - 3]]], dtype=torch.int32, device="cuda")
    width = 128 // (1 if fmt == F8 else 2)
    pools = [torch.zeros((n, 16, width), dtype=torch.uint8, device="cuda") for _ in range(2)]
    blocks = [torch.zeros((n, 16, 4), dtype=torch.uint8, device="cuda") for _ in range(2)] if fmt == MX else [None, None]
    cache = zc.PagedCache(pools[0], pools[1], table, torch.tensor([30], dtype=torch.int32, device="cuda"), fmt, None, None, *blocks)
    k, v = rows(30, 2, 128)
    zc.write_kv(k, v, cache, starts([30]))
    got = zc.read_kv(cache, starts([30]), 30)
    near = Pages([30], 2, 128, fmt)
    zc.write_kv(k, v, near.paged, starts([30]))
    want = zc.read_kv(near.paged, starts([30]), 30)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    touched = set(table.flatten().tolist())
    for pool in pools:                                           # nothing lies where offsets cut to 32 bits would write
        some = (pool.view(n, -1) != 0).any(dim=1).nonzero().flatten().tolist()
        assert set(some) <= touched


@pytest.mark.parametrize("fmt", FORMATS)
def test_results_with_strides(fmt):
    pages = Pages([40, 9], 2, 128, fmt)
    write_and_check(pages, [40, 9])
    k, v = zc.read_kv(pages.paged, starts([40, 9]), 49)
    room = torch.zeros((49, 6, 136), dtype=torch.bfloat16, device="cuda")
    zc.read_kv(pages.paged, starts([40, 9]), k=room[:, 0:4:2, :128], v=room[:, 1:5:2, :128])
    the_same(room[:, 0:4:2, :128].contiguous(), k, "k")
    the_same(room[:, 1:5:2, :128].contiguous(), v, "v")
    assert not bool(room[:, 4:].any()) and not bool(room[:, :, 128:].any())


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_step_recorded_and_replayed(fmt):
    """lengths += 1, write, attend, with the token's rows in buffers that change: a graph of it gives what the calls give."""
    heads, group, dim, steps = 2, 4, 128, 40
    lens = [15, 31, 0]
    a, b = (Pages([n + steps for n in lens], heads, dim, fmt, scales=fmt != BF16) for _ in range(2))
    k0, v0 = rows(sum(lens), heads, dim)
    for p in (a, b):
        p.lengths.copy_(torch.tensor(lens, dtype=torch.int32, device="cuda"))
        zc.write_kv(k0, v0, p.paged, starts(lens))
    bufs = [torch.zeros((3, heads * n, dim), dtype=torch.bfloat16, device="cuda") for n in (group, 1, 1)]
    out, lse = torch.zeros_like(bufs[0]), torch.zeros((3, heads * group), device="cuda")

    def step(p, o, z):
        p.lengths.add_(1)
        zc.write_kv(bufs[1], bufs[2], p.paged)
        zc.attend(bufs[0], p.paged, out=o, lse=z)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                                # (a first run outside of the capture, on a cache of its own)
        step(Pages([5, 5, 5], heads, dim, fmt, scales=fmt != BF16), torch.empty_like(out), torch.empty_like(lse))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, out, lse)
    g = gen(11)
    for i in range(steps):
        for x in bufs:
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        graph.replay()
        want, want_lse = torch.empty_like(out), torch.empty_like(lse)
        step(b, want, want_lse)
        if i % 13 == 0:
            torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse), i
    assert a.lengths.tolist() == [n + steps for n in lens]
    n = [x + steps for x in lens]
    for x, y in zip(zc.read_kv(a.paged, starts(n), sum(n)), zc.read_kv(b.paged, starts(n), sum(n))):
        assert torch.equal(x, y)


def test_another_stream_than_the_default_one():
    pages = Pages([64] * 4, 2, 128, MX)
    k, v = rows(4 * 64, 2, 128)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        zc.write_kv(k, v, pages.paged, starts([64] * 4))
        got = zc.read_kv(pages.paged, starts([64] * 4), 256)
    s.synchronize()
    want = quantised(k.to(torch.float32), MX)
    the_same(got[0], numbers(*want, MX, None), "k")
