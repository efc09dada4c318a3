#!/usr/bin/env python3
"""A K/V cache's life on one MI355X: compressed in pages, decoded, read by attention, and cut down by attention weight.

    python examples/kv_cache.py [--prompt 4096] [--answers 16] [--steps 24] [--keep 1024]

1. The cache of a long prompt lies compressed (FP8 pages of 16 tokens, one container for K and one for V); its pages are decoded.
2. Several answers are written under it: at every step zc.write_kv quantises each answer's new token into pages of its own, and
   zc.attend_shared reads the prompt's pages once for all of them.
3. One conversation goes on for longer: zc.attend with a window and sinks, keeping account of every token's attention weight.
4. zc.evict leaves the tokens that mattered; they are compressed again with the code that the prompt's pages were compressed with.
5. The conversation's whole cache goes to 4 bits: zc.read_kv reads it, zc.write_kv quantises it into MXFP4 pages, which attention reads as
   they are and the codec compresses with their block scales.

The "model" is random projections: the example is about the calls and who owns which memory."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2508_19263_amd import workloads as wl  # noqa: E402
from paper_2508_19263_amd import zc  # noqa: E402

HEADS, GROUP, DIM, PAGE = 8, 4, 128, 16


class Cache:
    """Pools and table of a batch's own cache, with room for `tokens` tokens per sequence, and append()."""

    def __init__(self, seqs, tokens, fmt=zc.FMT_FP8_E4M3, scale_k=None, scale_v=None):
        pages, block = -(-tokens // PAGE), zc.scale_block(fmt)
        n = seqs * HEADS * pages
        self.k = torch.zeros((n, PAGE, DIM * zc.elem_bits(fmt) // 8), dtype=torch.uint8, device="cuda")
        self.v = torch.zeros_like(self.k)
        self.k_blocks, self.v_blocks = (torch.zeros((n, PAGE, DIM // block), dtype=torch.uint8, device="cuda") if block else None for _ in range(2))
        self.table = torch.arange(n, dtype=torch.int32, device="cuda").view(seqs, HEADS, pages)
        self.lengths = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        scales = [None if x is None else x.expand(seqs, HEADS).contiguous() for x in (scale_k, scale_v)]
        self.paged = zc.PagedCache(self.k, self.v, self.table, self.lengths, fmt, *scales, self.k_blocks, self.v_blocks)

    def append(self, k, v):
        """One token per sequence: k, v BF16 [seqs, heads, dim]."""
        self.lengths += 1                                        # (a length counts the tokens that are being written)
        zc.write_kv(k, v, self.paged)


def main(prompt=4096, answers=16, steps=24, keep=1024, quiet=False):
    def say(*x):
        if not quiet:
            print(*x, flush=True)

    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    keep = min(keep, prompt)

    # ---- 1. the prompt's pages, compressed; their code; decoded
    k, v = wl.fp8_kv_pair(1, HEADS, prompt, DIM, "cuda", seed=5)
    params = zc.params(zc.FMT_FP8_E4M3, PAGE * DIM, streams=8, flags=zc.FLAG_REVERSE_FIELDS)
    codes = [zc.train_code(x, x.numel(), params) for x in (k, v)]
    packed = [zc.compress_with_code(x, x.numel(), params, c) for x, c in zip((k, v), codes)]
    say("prompt of %d tokens: %.2f MB of pages, %.2f MB compressed" % (prompt, 2 * k.numel() / 1e6, sum(c.numel() for c, _ in packed) / 1e6))
    pools = [zc.decompress(c, info)[0].view(-1, PAGE, DIM) for c, info in packed]
    assert torch.equal(pools[0].view(-1), k.view(-1)) and torch.equal(pools[1].view(-1), v.view(-1))
    scale_k, scale_v = torch.full((1, HEADS), 45.0 / 448, device="cuda"), torch.full((1, HEADS), 5.0 / 448, device="cuda")
    table = torch.arange(pools[0].shape[0], dtype=torch.int32, device="cuda").view(1, HEADS, -1)
    length = torch.full((1,), prompt, dtype=torch.int32, device="cuda")
    shared = zc.PagedCache(pools[0], pools[1], table, length, zc.FMT_FP8_E4M3, scale_k, scale_v)

    # ---- 2. answers under it, one token each at a time
    own = Cache(answers, steps, zc.FMT_FP8_E4M3, scale_k, scale_v)
    mix = torch.randn((DIM, 3 * DIM), generator=g, device="cuda") / DIM ** 0.5
    x = torch.randn((answers, HEADS * GROUP, DIM), generator=g, device="cuda")
    for i in range(steps):
        q, nk, nv = (x @ mix).to(torch.bfloat16).split(DIM, dim=-1)
        own.append(nk[:, ::GROUP], nv[:, ::GROUP])
        out, lse = zc.attend_shared(q, shared, own.paged, max_kv_len=i + 1, max_prefix_len=prompt)
        x = torch.tanh(x + out.float())
    say("%d answers of %d tokens under it, lse %.3f .. %.3f" % (answers, steps, lse.min().item(), lse.max().item()))

    # ---- 3. a conversation over the same pages: all of it is seen, and account is kept
    weights = torch.zeros((1, HEADS, shared.capacity), device="cuda")
    for i in range(steps):
        q = torch.randn((1, HEADS * GROUP, DIM), generator=g, device="cuda").to(torch.bfloat16)
        zc.attend(q, shared, weights=weights, weights_out=weights)
    near, _ = zc.attend(q, shared, window=keep, sinks=4)
    say("attention weight of %d steps: %.1f per head" % (steps, weights.sum().item() / HEADS))

    # ---- 4. what stays
    small = Cache(1, keep, zc.FMT_FP8_E4M3, scale_k, scale_v)
    left = torch.zeros((1, HEADS, small.paged.capacity), device="cuda")
    kept = zc.evict(shared, weights, keep, small.paged, left, sinks=4, recent=keep // 4)
    full, _ = zc.attend(q, shared)
    rest, _ = zc.attend(q, small.paged)
    again = [zc.compress_with_code(x, x.numel(), params, c) for x, c in zip((small.k, small.v), codes)]
    back = [zc.decompress(c, info)[0] for c, info in again]
    assert torch.equal(back[0], small.k.view(-1)) and torch.equal(back[1], small.v.view(-1))
    share = left.sum().item() / weights.sum().item()
    off = ((rest.float() - full.float()).norm() / full.float().norm()).item()
    say("%d of %d tokens stay with %.0f %% of the weight: %.2f MB of pages, %.2f MB compressed; attention over them is %.3f off"
        % (keep, prompt, 100 * share, 2 * small.k.numel() / 1e6, sum(c.numel() for c, _ in again) / 1e6, off))

    # ---- 5. all of it in 4 bits
    whole = torch.tensor([0, prompt], dtype=torch.int32, device="cuda")
    keys, values = zc.read_kv(shared, whole, prompt)
    four = Cache(1, prompt, zc.FMT_FP4_E2M1_MX)
    four.lengths.fill_(prompt)
    zc.write_kv(keys, values, four.paged, whole)
    coarse, _ = zc.attend(q, four.paged)
    params4 = zc.params(zc.FMT_FP4_E2M1_MX, PAGE * DIM // 2, streams=8)
    packed4 = [zc.compress(x, x.numel() * 2, params4, scales=b) for x, b in ((four.k, four.k_blocks), (four.v, four.v_blocks))]
    for (c, info), x, b in zip(packed4, (four.k, four.v), (four.k_blocks, four.v_blocks)):
        bits, blocks = zc.decompress(c, info)
        assert torch.equal(bits.view(-1), x.view(-1)) and torch.equal(blocks.view(-1), b.view(-1))
    off4 = ((coarse.float() - full.float()).norm() / full.float().norm()).item()
    say("in 4 bits: %.2f MB of pages and scales, %.2f MB compressed; attention over them is %.3f off"
        % (2 * (four.k.numel() + four.k_blocks.numel()) / 1e6, sum(c.numel() for c, _ in packed4) / 1e6, off4))
    return {"coarse": coarse, "kept": kept, "share": share, "out": out, "near": near, "rest": rest, "full": full, "lengths": small.lengths}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--prompt", type=int, default=4096)
    ap.add_argument("--answers", type=int, default=16)
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--keep", type=int, default=1024)
    a = ap.parse_args()
    if a.prompt % PAGE:
        ap.error("--prompt has to be a multiple of %d" % PAGE)
    main(a.prompt, a.answers, a.steps, a.keep)
