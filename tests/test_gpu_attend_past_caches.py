"""Attention whose pages may go past the caches, which the lengths and the table decide on the device: on both sides of that decision the same bits, and
those of the definition in 64 bits."""
import pytest
import torch

from paper_2508_19263_amd import zc
from tests.paged import Cache, agree, gen, starts
from tests.test_gpu_attend import check, queries

pytestmark = pytest.mark.gpu

BF16, E4M3, E5M2 = zc.FMT_BF16, zc.FMT_FP8_E4M3, zc.FMT_FP8_E5M2
HELD = 256 << 20                                               # bytes of the memory-side cache


class Big:
    """A cache of random pages of more than HELD bytes; `tokens` of all sequences are what HELD has."""

    def __init__(self, fmt, dim, heads, seqs, length, page=16, seed=1):
        g, width = gen(seed), 2 if fmt == BF16 else 1
        self.tokens, self.length, self.fmt = HELD // (2 * heads * dim * width), length, fmt
        per = -(-length // page)
        n = seqs * heads * per + 3
        assert n * page * dim * width * 2 > HELD and seqs * length > self.tokens
        pools = []
        for _ in range(2):
            x = torch.randn((n, page, dim), generator=g, device="cuda", dtype=torch.float32)
            pools.append(x.to({BF16: torch.bfloat16, E4M3: torch.float8_e4m3fn, E5M2: torch.float8_e5m2}[fmt]))
        self.table = torch.randperm(n, generator=g, device="cuda")[:n - 3].view(seqs, heads, per).to(torch.int32)
        self.lengths = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        self.pools, self.page = pools, page
        self.paged = zc.PagedCache(pools[0], pools[1], self.table, self.lengths, fmt)

    def set(self, lens):
        self.lengths.copy_(torch.tensor(lens, dtype=torch.int32))

    def rows(self, seq, head):
        """K and V of one head in 64 bits."""
        n = int(self.lengths[seq])
        return [x[self.table[seq, head].long()].flatten(0, 1)[:n].to(torch.float64) for x in self.pools]


def close(big, q, out, lse, seqs):
    """Single tokens of some sequences against the definition, with the tolerances of tests.paged.attention."""
    heads, dim = big.table.shape[1], q.shape[2]
    group, bits = q.shape[1] // heads, 2.0 ** -9 if big.fmt == BF16 else 2.0 ** -12
    for s in seqs:
        for h in range(heads):
            k, v = big.rows(s, h)
            mine = slice(h * group, (h + 1) * group)
            x = q[s, mine].to(torch.float64)
            logits = (x @ k.t()) * dim ** -0.5
            z = torch.logsumexp(logits, 1, keepdim=True)
            p = torch.exp(logits - z)
            o, size = p @ v, ((x.abs() @ k.abs().t()) * dim ** -0.5).amax(1, keepdim=True)
            d, sums = dim * 2.0 ** -24 * size + 2.0 ** -22 * (1 + size), k.shape[0] * 2.0 ** -24
            agree(out[s, mine], o, 2 * (2.0 ** -8 * o.abs() + (bits + 2 * d + sums) * (p @ v.abs()) + 2.0 ** -24), "out")
            agree(lse[s, mine], z.squeeze(1), (2 * (d + sums + 2.0 ** -22 * (1 + z.abs()))).squeeze(1), "lse")


@pytest.mark.parametrize("fmt,dim,group", [(BF16, 128, 1), (BF16, 64, 4), (E4M3, 128, 4), (E5M2, 64, 20)])
@pytest.mark.parametrize("seqs,heads", [(5, 8), (70, 2)])
def test_lengths_on_both_sides(fmt, dim, group, seqs, heads):
    width = 2 if fmt == BF16 else 1
    need = HELD // (2 * heads * dim * width)                   # tokens that the caches hold
    length = need // seqs + 700
    big = Big(fmt, dim, heads, seqs, length)
    q = queries(seqs, heads * group, dim)
    kept = {}
    for total in (need + 2 * seqs, need, need - 2 * seqs, need // 3):          # more, as many, less: the first sequence has the same length in all
        rest = total - length
        lens = [length] + [rest // (seqs - 1) + (1 if i < rest % (seqs - 1) else 0) for i in range(seqs - 1)]
        assert sum(lens) == total and max(lens) <= length
        big.set(lens)
        out, lse = zc.attend(q, big.paged)
        print("case", fmt, dim, seqs, total, flush=True)
        for name, x in (("out", out), ("lse", lse)):
            assert torch.equal(x[0], kept.setdefault(name, x[0].clone())), name
        close(big, q, out, lse, (0, seqs - 1))


@pytest.mark.parametrize("fmt,dim", [(BF16, 128), (E4M3, 64)])
@pytest.mark.parametrize("seqs,heads", [(5, 8), (66, 2)])
def test_pages_of_several_sequences(fmt, dim, seqs, heads):
    """Sequences that have pages in common give what copies of them do: none, a part, the middle, all; with the same queries the same bits."""
    width = 2 if fmt == BF16 else 1
    length = HELD // (2 * heads * dim * width) // seqs + 300
    big = Big(fmt, dim, heads, seqs, length)
    big.set([length] * seqs)
    q = queries(seqs, heads * 4, dim)
    own = big.table.clone()
    for part in (0.0, 0.3, 0.7, 1.0):
        n = int(part * big.table.shape[2])
        big.table.copy_(own)
        big.table[:, :, :n] = own[:1, :, :n]
        out, lse = zc.attend(q, big.paged)
        close(big, q, out, lse, (0, seqs - 1))
        if part == 1.0:
            q2 = q[:1].expand_as(q).contiguous()
            out, lse = zc.attend(q2, big.paged)
            assert torch.equal(out, out[:1].expand_as(out)) and torch.equal(lse, lse[:1].expand_as(lse))
            big.set([length] + [0] * (seqs - 1))
            one, one_lse = zc.attend(q2, big.paged)
            assert torch.equal(one[0], out[0]) and torch.equal(one_lse[0], lse[0])
            assert bool((one[1:] == 0).all()) and bool((one_lse[1:] == -float("inf")).all())


@pytest.mark.parametrize("window", [0, 3000])
def test_windows_weights_rows_and_absent_pages(window):
    seqs, heads, dim = 9, 8, 128
    length = HELD // (2 * heads * dim * 2) // seqs + 500
    big = Big(BF16, dim, heads, seqs, length)
    q_lens = [3] * seqs
    q = queries(3 * seqs, heads * 4, dim)
    many = dict(q_start=starts(q_lens), max_q_len=3, window=window, sinks=5 if window else 0)
    kept = []
    for lens in ([length] * seqs, [length, 40] + [0] * (seqs - 2), [length, 40, 3] + [length] * (seqs - 3)):
        big.set(lens)
        w = torch.zeros((seqs, heads, big.paged.capacity), device="cuda")
        out, lse = zc.attend(q, big.paged, weights_out=w, **many)
        plain, plain_lse = zc.attend(q, big.paged, **many)
        assert torch.equal(out, plain) and torch.equal(lse, plain_lse)
        kept.append((out[:3].clone(), lse[:3].clone(), w[0].clone()))
        assert all(torch.equal(a, b) for a, b in zip(kept[0], kept[-1]))
        # each of a head's 12 rows gives 1 in all; |logits| add up to less than 16, so weights are off by (128 * 16 + 4 * 17) * 2^-24, twice, and sums by 7,782 * 2^-24
        assert bool(((w[0].sum(1, dtype=torch.float64) - 12).abs() < 12 * 2 * (2 * 2116 + 7782) * 2.0 ** -24).all())
    big.table[0, 0, big.table.shape[2] // 2] = -1              # the page that is looked at
    big.set([length] * seqs)
    out, _ = zc.attend(q, big.paged, **many)
    big.set([length] + [0] * (seqs - 1))
    again, _ = zc.attend(q, big.paged, **many)
    assert torch.equal(out[:3], again[:3]) and bool(out[:3].isfinite().all())


@pytest.mark.parametrize("fmt", [BF16, E4M3])
def test_a_recorded_step_goes_by_the_lengths_of_its_replay(fmt):
    seqs, heads, dim = 6, 8, 128
    length = HELD // (2 * heads * dim * (2 if fmt == BF16 else 1)) // seqs + 200
    big = Big(fmt, dim, heads, seqs, length)
    big.set([100] * seqs)
    q = queries(seqs, heads * 4, dim)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    zc.attend(q, big.paged, out=out, lse=lse, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        zc.attend(q, big.paged, out=out, lse=lse, ws=ws)
    for lens in ([length] * seqs, [100] * seqs, [length] * (seqs - 1) + [0], [0] * seqs, [length] * seqs):
        big.set(lens)
        graph.replay()
        want, want_lse = zc.attend(q, big.paged)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_a_pool_that_the_caches_hold():
    """Much room over a small pool: the tables name its pages many times."""
    cache = Cache([300, 1, 0, 1037, 64, 4099, 16, 17], 8, 128, BF16)
    room = torch.full((8, 8, 40000 // 16), -1, dtype=torch.int32, device="cuda")
    room[:, :, :cache.table.shape[2]] = cache.table
    p = cache.paged
    cache.table, cache.paged = room, zc.PagedCache(p.k_pages, p.v_pages, room, cache.lengths, BF16)
    check(cache, [1] * 8, 4, 0, 0, weights=True)


@pytest.mark.parametrize("length", [767, 768, 800])
def test_many_short_caches(length):
    """Parts on both sides of what is worth choosing for; more sequences than are looked at."""
    heads, dim = 2, 128
    seqs = HELD // (2 * heads * dim * 2) // 700
    big = Big(BF16, dim, heads, seqs, length + 33)
    q = queries(seqs, heads * 4, dim)
    lens = [length, 1, 0] + [length + (i % 67) - 33 for i in range(seqs - 3)]
    big.set(lens)
    out, lse = zc.attend(q, big.paged)
    close(big, q, out, lse, (0, 1, 3, 36, 37, seqs // 2, seqs - 1))
    assert bool((out[2] == 0).all())
    half = [n if i % 300 == 0 else 0 for i, n in enumerate(lens)]
    big.set(half)
    again, again_lse = zc.attend(q, big.paged)
    on = torch.tensor([n > 0 for n in half], device="cuda")
    assert torch.equal(again[on], out[on]) and torch.equal(again_lse[on], lse[on]) and bool((again[~on] == 0).all())
