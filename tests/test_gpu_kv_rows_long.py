"""Calls of zc.write_kv and zc.read_kv that are large enough for their workgroups to take four times as many tokens: stored bits, and rows read
back, are those of the definition (tests/paged4.py), everything else is as it was."""
import pytest
import torch

from paper_2508_19263_amd import zc
from tests.paged import gen, starts
from tests.paged4 import MX, NV
from tests.test_gpu_kv_rows import BF16, F8, FORMATS, Pages, compare, numbers, quantised, rows, the_same

pytestmark = pytest.mark.gpu

# tokens of 16 heads whose workgroups of 256 threads, a row to every dim / 8 of them, are 2,048 and a few
MANY = {64: 128 * 32 + 33, 128: 128 * 16 + 17}
HEADS = 16


def ragged(n, most, seed):
    """Numbers of tokens of sequences, n in all, none of a sequence among them."""
    g, lens = torch.Generator().manual_seed(seed), []
    while sum(lens) < n:
        lens.append(min(int(torch.randint(0, most + 1, (1,), generator=g)), n - sum(lens)))
    return lens + [0]


def where(pages, start, n):
    """Of every token: its sequence (-1: none), and per head the page (-1: none) and the place in it."""
    t = torch.arange(n, device="cuda")
    begins = start.to(torch.int64)
    seq = torch.searchsorted(begins, t, right=True) - 1
    ours = (seq >= 0) & (seq < len(pages.lens))
    seq = torch.where(ours, seq, torch.zeros_like(seq))
    at = pages.lengths.to(torch.int64)[seq] - (begins[seq + 1] - t)
    inside = ours & (at >= 0) & (at < pages.table.shape[2] * pages.page)
    at = torch.where(inside, at, torch.zeros_like(at))
    page = pages.table.to(torch.int64)[seq, :, at // pages.page]
    there = inside.view(-1, 1) & (page >= 0) & (page < pages.pools["k"].shape[0])
    return ours, seq, torch.where(there, page, torch.full_like(page, -1)), (at % pages.page).view(-1, 1).expand_as(page)


def after_write(pages, k, v, start):
    pools = {name: x.clone() for name, x in pages.pools.items()}
    _, seq, page, slot = where(pages, start, k.shape[0])
    there = page >= 0
    for name, x in (("k", k), ("v", v)):
        y = x.to(torch.float32)
        if pages.scales[name] is not None:
            scale, most = pages.scales[name][seq].unsqueeze(2), torch.finfo(torch.float32).max
            y = torch.where(scale == 0, torch.zeros_like(y), y * (1.0 / scale).clamp(-most, most))
        bits, blocks = quantised(y, pages.fmt)
        if pages.fmt == BF16 and pages.scales[name] is None:
            bits = x.contiguous().view(torch.int16)
        pools[name][page[there], slot[there]] = bits[there]
        if blocks is not None:
            pools[name + "_blocks"][page[there], slot[there]] = blocks[there]
    return pools


def check_read(pages, start, n, room):
    """room: K and V with what they hold before."""
    ours, seq, page, slot = where(pages, start, n)
    there = (page >= 0).unsqueeze(2)
    before = [x.clone() for x in room]
    zc.read_kv(pages.paged, start, k=room[0], v=room[1])
    for name, got, was in zip("kv", room, before):
        blocks = pages.pools.get(name + "_blocks")
        page0 = page.clamp(min=0)
        scale = None if pages.scales[name] is None else pages.scales[name][seq].unsqueeze(2)
        want = numbers(pages.pools[name][page0, slot], None if blocks is None else blocks[page0, slot], pages.fmt, scale)
        want = torch.where(there, want, torch.zeros_like(want))
        the_same(got.contiguous(), torch.where(ours.view(-1, 1, 1), want, was), name)


def check(pages, start, n, wide=False, k=None, v=None):
    if k is None:
        k, v = rows(n, pages.heads, pages.dim, wide=wide)
    want = after_write(pages, k, v, start)
    zc.write_kv(k, v, pages.paged, start)
    torch.cuda.synchronize()
    compare(pages, want)
    room = torch.full((n, pages.heads * 2 + 1, pages.dim + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    check_read(pages, start, n, (room[:, 1::2, :pages.dim], room[:, :-1:2, :pages.dim]) if wide else [torch.full_like(k, 3.0) for _ in "kv"])
    if wide:
        assert bool((room[:, -1, pages.dim:] == 3).all()) and bool((room[:, :, pages.dim:] == 3).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scales", [False, True])
@pytest.mark.parametrize("most", [1, 40, 700, 10000])
def test_sequences_of_many_lengths(fmt, dim, scales, most):
    """A token or none to a sequence (more sequences than are counted one by one), tens, hundreds, all of one."""
    n = MANY[dim]
    q_lens = ragged(n, most, dim + most)
    pages = Pages([x + (i * 13) % 20 for i, x in enumerate(q_lens)] if most > 1 else [x + i % 3 for i, x in enumerate(q_lens)], HEADS, dim, fmt, scales=scales)
    assert most > 1 or len(q_lens) > 1024
    check(pages, starts(q_lens), n, wide=most == 40)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
def test_tokens_without_a_sequence_or_a_page(fmt, dim):
    """Tokens before the first sequence and behind the last, pages that are absent, lengths past the table's room and less than what is written."""
    n = MANY[dim]
    q_lens = [n // 3, 0, 41, n // 3, 200]
    start = starts(q_lens) + 29
    pages = Pages([n // 3 + 5, 100, 41, n // 3, 210], HEADS, dim, fmt, page=32, scales=fmt == NV)
    pages.table[0, ::2, 3:9] = -1
    pages.table[3, 5] = pages.paged.n_pages
    room = pages.table.shape[2] * pages.page
    for seq, length in ((0, room + 3), (2, 7), (4, -1)):
        pages.lengths[seq] = pages.lens[seq] = length
    check(pages, start, n, wide=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_numbers_of_every_kind(fmt):
    """All BF16 numbers in random order, without scales and with ones of every size and kind."""
    n = MANY[128] - 1 + 16
    every = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16).view(torch.bfloat16)
    order = torch.cat([torch.randperm(65536, generator=gen(i), device="cuda") for i in range(n * HEADS * 128 // 65536 + 1)])[:n * HEADS * 128]
    x = every[order].view(n, HEADS, 128)
    finite = torch.where(x.isfinite(), x, torch.zeros_like(x))
    for k, v in ((x, finite), (finite, x.flip(0))):
        check(Pages([n], HEADS, 128, fmt), starts([n]), n, k=k, v=v)
        q_lens = [n // 8] * 7 + [n - n // 8 * 7]
        pages = Pages(q_lens, HEADS, 128, fmt, scales=True)
        for i, name in enumerate("kv"):
            s = torch.exp2(torch.randint(-140, 128, (8, HEADS), generator=gen(i + 90), device="cuda").to(torch.float32)) * pages.scales[name]
            s[1], s[2, ::2], s[3], s[4, 1::2] = -s[1], 0.0, float("inf"), float("nan")
            pages.scales[name].copy_(s)
        check(pages, starts(q_lens), n, k=k, v=v)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
def test_large_and_small_calls_agree(fmt, dim):
    """The same tokens in one call and in many, a token to each sequence in the last one."""
    n, seqs = MANY[dim] // 8 * 8, 8
    a, b = (Pages([n // seqs] * seqs, HEADS, dim, fmt, scales=True) for _ in range(2))
    k, v = rows(n, HEADS, dim)
    zc.write_kv(k, v, a.paged, starts([n // seqs] * seqs))
    view = [x.view(seqs, n // seqs, HEADS, dim) for x in (k, v)]
    for first, last in ((0, 1), (1, n // seqs - 1)):
        b.lengths.fill_(last)
        zc.write_kv(*[x[:, first:last].reshape(-1, HEADS, dim) for x in view], b.paged, starts([last - first] * seqs))
    b.lengths.fill_(n // seqs)
    zc.write_kv(*[x[:, -1] for x in view], b.paged)
    compare(b, a.pools)
    whole = zc.read_kv(a.paged, starts([n // seqs] * seqs), n)
    last = zc.read_kv(a.paged)
    for x, y in zip(whole, last):
        assert torch.equal(x.view(seqs, -1, HEADS, dim)[:, -1], y)


@pytest.mark.parametrize("fmt", [F8, MX, NV])
def test_recorded_and_replayed(fmt):
    n = MANY[128]
    q_lens = ragged(n, 300, 5)
    pages = Pages([x + 3 for x in q_lens], HEADS, 128, fmt, scales=fmt != MX)
    k, v = rows(n, HEADS, 128)
    start = starts(q_lens)
    back = [torch.zeros_like(x) for x in (k, v)]
    zc.write_kv(k, v, pages.paged, start)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        zc.write_kv(k, v, pages.paged, start)
        zc.read_kv(pages.paged, start, k=back[0], v=back[1])
    for i in range(4):
        k.copy_(torch.randn(k.shape, generator=gen(i), device="cuda"))
        v.copy_(torch.randn(v.shape, generator=gen(i + 50), device="cuda"))
        want = after_write(pages, k, v, start)
        graph.replay()
        if i % 2:
            torch.cuda.synchronize()
        compare(pages, want)
        for x, y in zip(zc.read_kv(pages.paged, start, n), back):
            assert torch.equal(x, y)


def test_these_calls_are_large():
    """As many workgroups as take four times as many tokens, the last of them not full."""
    for dim, n in MANY.items():
        each = 256 // (dim // 8)
        assert -(-n // each) * HEADS >= 2048 and n % (each * 4)
