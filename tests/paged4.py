"""Caches in pages of 4 bits for the tests, their elements and what quantising means, in 64 bits and written from the definitions."""
import math

import torch

from paper_2508_19263_amd import zc
from tests.paged import gen

MX, NV = zc.FMT_FP4_E2M1_MX, zc.FMT_FP4_E2M1_NV
BLOCK = {MX: 32, NV: 16}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def small_float(mantissa, least):
    """All non-negative numbers of a small float type below its largest exponent's end, by code."""
    numbers = []
    for code in range(128):
        e, m = code >> mantissa, code & ((1 << mantissa) - 1)
        numbers.append(2.0 ** least * m / (1 << mantissa) if e == 0 else 2.0 ** (least + e - 1) * (1 + m / (1 << mantissa)))
    return numbers


E4M3 = small_float(3, -6)[:127]                                  # to 448; 127 is NaN
E5M2 = small_float(2, -14)[:124]                                 # to 57344


def nearest(y, grid):
    """Codes of the numbers of an ascending grid (even codes: even mantissas) next to |y|, ties to even, the last one beyond it; float64 y."""
    g = torch.tensor(grid, dtype=torch.float64, device=y.device)
    a = y.abs().clamp(max=grid[-1])
    hi = torch.searchsorted(g, a).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    below, above = a - g[lo], g[hi] - a
    return torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)


def scale_value(blocks, fmt):
    """Block scales' bytes -> float64."""
    b = blocks.to(torch.int64) & 255
    if fmt == MX:
        return torch.where(b == 255, torch.full(b.shape, math.nan, dtype=torch.float64, device=b.device), torch.exp2((b - 127).to(torch.float64)))
    table = torch.tensor(E4M3 + [math.nan], dtype=torch.float64, device=b.device)
    return torch.where(b >= 128, -table[b & 127], table[b & 127])


def element_value(bits):
    """Packed elements [..., dim / 2] -> float64 [..., dim], without their blocks' scales."""
    code = torch.stack([bits & 15, (bits >> 4) & 15], dim=-1).flatten(-2).to(torch.int64)
    x = torch.tensor(GRID, dtype=torch.float64, device=bits.device)[code & 7]
    return torch.where(code >= 8, -x, x)


def values4(bits, blocks, fmt):
    x = element_value(bits).unflatten(-1, (-1, BLOCK[fmt]))
    return (x * scale_value(blocks, fmt).unsqueeze(-1)).flatten(-2)


def quantised4(y, fmt):
    """float32 [..., dim] -> (packed elements, block scales), as zc_kv_write's definition says."""
    y = y.to(torch.float64).unflatten(-1, (-1, BLOCK[fmt]))
    nan = y.isnan().any(dim=-1, keepdim=True)
    most = float(torch.finfo(torch.float32).max)
    m = y.nan_to_num(0.0, most, -most).abs().amax(dim=-1, keepdim=True)
    if fmt == MX:
        e = torch.where(m > 0, torch.frexp(m).exponent - 3, torch.full(m.shape, -127, dtype=torch.int32, device=m.device)).clamp(min=-127)
        blocks, s = e + 127, torch.exp2(e.to(torch.float64))
        blocks = torch.where(nan, torch.full_like(blocks, 255), blocks)
    else:
        blocks = nearest((m.to(torch.float32) / 6.0).to(torch.float64), E4M3)
        s = scale_value(blocks, NV)
        blocks = torch.where(nan, torch.full_like(blocks, 127), blocks)
    # the number times s that is next to y: distances of products, which 64 bits hold exactly
    flat, steps = y.nan_to_num(0.0, most, -most), [g * s for g in GRID]
    code = torch.zeros(flat.shape, dtype=torch.int64, device=y.device)
    for i in range(1, 8):
        half = (steps[i - 1] + steps[i]) / 2
        code += (flat.abs() > half) | ((flat.abs() == half) & (i % 2 == 0))
    code = torch.where(nan | (s == 0), torch.zeros_like(code), code + 8 * torch.signbit(y).to(torch.int64)).flatten(-2)
    return (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8), blocks.squeeze(-1).to(torch.uint8)


class Cache4:
    """As tests.paged.Cache, in a format of 4 bits: `k`, `v` are its numbers [seqs, heads, tokens, dim] in 64 bits (without the scales per sequence
    and head), `bits` and `blocks` what is stored of them; what no token of a sequence lies in holds NaN.  `fmt` is the format whose weights
    attention rounds to the same type, which is what paged.attention goes by; `format` the cache's own."""

    def __init__(self, lens, heads, dim, fmt, page=16, seed=1, spare_pages=3, room=None, edit=None, scales=None):
        g = gen(seed)
        seqs, self.lens, self.page, self.format = len(lens), list(lens), page, fmt
        self.fmt = zc.FMT_BF16 if fmt == MX else zc.FMT_FP8_E4M3
        pages = max(1, -(-max(list(lens) + [room or 0]) // page))
        shape = (seqs, heads, pages * page, dim)
        self.bits, self.blocks = {}, {}
        for name in "kv":
            x = torch.randn(shape, generator=g, device="cuda")
            if name == "k":
                x[..., :: max(1, dim // 4)] *= 6.0
            x *= torch.exp2(torch.randint(-3, 4, shape[:3] + (1,), generator=g, device="cuda").to(torch.float32) / (4.0 if name == "k" else 1.0))
            self.bits[name], self.blocks[name] = quantised4(x, fmt)
        if edit:
            edit(self)
        self.k, self.v = (values4(self.bits[name], self.blocks[name], fmt) for name in "kv")
        if scales is None:
            scales = fmt == NV
        self.ks = torch.rand((seqs, heads), generator=g, device="cuda") + 0.5 if scales else None
        self.vs = torch.rand((seqs, heads), generator=g, device="cuda") + 0.5 if scales else None
        self.lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
        used = seqs * heads * pages
        order = torch.randperm(used + spare_pages, generator=g, device="cuda")[:used]
        self.table = order.view(seqs, heads, pages).to(torch.int32)
        inside = (torch.arange(pages * page, device="cuda") < self.lengths.view(-1, 1)).view(seqs, 1, -1, 1)
        self.pools = {}
        for name in "kv":
            for kind, x, junk in (("", self.bits[name], 0xFF), ("_blocks", self.blocks[name], 0xFF if fmt == MX else 0x7F)):
                pool = torch.full((used + spare_pages, page, x.shape[-1]), junk, dtype=torch.uint8, device="cuda")
                pool[order] = torch.where(inside, x, torch.full_like(x, junk)).view(used, page, x.shape[-1])
                self.pools[name + kind] = pool
        self.paged = zc.PagedCache(self.pools["k"], self.pools["v"], self.table, self.lengths, fmt, self.ks, self.vs, self.pools["k_blocks"], self.pools["v_blocks"])

    def rows(self, name, seq, head):
        """Numbers times the scale of sequence and head, [tokens, dim] in 64 bits."""
        x = getattr(self, name)[seq, head, :self.lens[seq]]
        scale = getattr(self, name + "s")
        return x if scale is None else x * scale[seq, head].to(torch.float64)

    def present(self, seq, head):
        ok = (self.table[seq, head] >= 0) & (self.table[seq, head] < self.paged.n_pages)
        return ok.repeat_interleave(self.page)[:self.lens[seq]]
