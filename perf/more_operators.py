"""A K/V cache in pages: quantised as it is written, read back, and attention over pages of 4 bits, as measurable cases.

A page is `page` tokens of one K/V head of one sequence, [page][dim] elements; a table gives the page of every stretch of
`page` tokens.  Pages of a pool lie in random order, tokens behind a sequence's end and pages that no table names hold
whatever was there before (NaN here).  Element formats:
  bf16, fp8 (E4M3), e5m2   FP8 with a float scale per sequence and head, which its elements are divided by when they are written
  mx   E2M1, two to a byte (the first in the low bits), with an E8M0 scale for every 32 elements of a token: 2^(floor(log2 of the largest) - 2)
  nv   E2M1 with an E4M3 scale for every 16 (the largest / 6) and a float scale per sequence and head
Elements are rounded to the nearest, ties to even, and what is beyond the largest number becomes that.
A case is a dict of plain values:
  op       "write" (the last q tokens of every sequence are quantised into its pages, and read back as attention will see them),
           "read" (the last q tokens of every sequence are read back), "attend" (attention with a sliding window and sinks over the
           whole cache), "shared" (the same for a batch that shares a prefix)
  fmt, seqs, heads, group, dim, page   element format, sequences, K/V heads, query heads per K/V head, head dimension, tokens per page
  kv_hi, kv_lo   lengths of the sequences' own caches, spread evenly from the one to the other
  q_hi, q_lo     tokens per sequence that are written, read or asked with, spread likewise; token i of n is at position len - n + i
  window, sinks  0: every earlier token is visible
  prefix   tokens of the shared prefix
  weights  1: the attention weight of every cached token is added up too

Where `own` is false the operators are computed from elementary torch operations in 32 bits, else by the library's kernels.
"""
import math

import torch

own = False

BLOCK = {"mx": 32, "nv": 16}                                     # elements that share a scale
LARGEST = {"fp8": 448.0, "e5m2": 57344.0, "nv": 6.0 * 448.0}     # what a scale per sequence and head maps the largest number to
FP8 = {"fp8": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TIES = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)                   # between neighbours of 0, 0.5, 1, 1.5, 2, 3, 4, 6


def _case(name, op, fmt, seqs, kv_hi, kv_lo, heads=8, group=4, dim=128, page=16, q_hi=1, q_lo=1, window=0, sinks=0, prefix=0, weights=0):
    c = dict(op=op, fmt=fmt, seqs=seqs, heads=heads, group=group, dim=dim, page=page, kv_hi=kv_hi, kv_lo=kv_lo, q_hi=q_hi, q_lo=q_lo,
             window=window, sinks=sinks, prefix=prefix, weights=weights)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the new token of every conversation of a server's batch: the smallest write, latency alone
        _case("write_tokens", "write", "mx", 32, 5003, 17),
        # pieces of three prompts behind what is cached of them, to FP8 pages with given scales
        _case("write_pieces", "write", "fp8", 3, 4111, 700, page=64, q_hi=1024, q_lo=333),
        # two whole prompts: the largest write
        _case("write_prompts", "write", "nv", 2, 16384, 15001, q_hi=16384, q_lo=15001),
        # a short conversation with small heads, for another machine
        _case("read_short", "read", "nv", 1, 777, 777, heads=4, dim=64, q_hi=777, q_lo=777),
        # a batch of long ones: the largest read
        _case("read_long", "read", "mx", 8, 20011, 1001, q_hi=20011, q_lo=1001),
        # the next token of one conversation: the smallest call, latency alone
        _case("decode_one", "attend", "mx", 1, 1000, 1000, window=512, sinks=4),
        # the next tokens of a batch whose caches fill a good part of the memory's bandwidth for a while
        _case("decode_batch", "attend", "mx", 32, 16384, 16384),
        # a batch at all stages, an empty slot among them, that keeps account of every token's weight
        _case("decode_ragged", "attend", "nv", 24, 30011, 0, weights=1),
        # five drafted tokens per sequence to be checked at once, small heads
        _case("decode_draft", "attend", "nv", 6, 7919, 3001, group=7, dim=64, q_hi=5, q_lo=5, window=2048, sinks=64),
        # a piece of two long prompts over what is cached of them already
        _case("prefill_chunk", "attend", "mx", 2, 9001, 8191, q_hi=1024, q_lo=511, window=4096, sinks=4),
        # a whole prompt: the largest call
        _case("prefill_long", "attend", "nv", 1, 8192, 8192, q_hi=8192, q_lo=8192),
        # many answers under one long document
        _case("shared_many", "shared", "mx", 64, 777, 16, prefix=32768),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(("write", "write", "read", "attend", "attend", "attend", "shared"))
    fmt = rng.choice(("mx", "nv") if op in ("attend", "shared") else ("mx", "nv", "mx", "nv", "fp8", "e5m2", "bf16"))
    heads, group, dim, page = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 3, 4, 5, 7, 8)), rng.choice((128, 128, 64)), rng.choice((16, 16, 32, 64))
    window = rng.choice((0, 0, _log_uniform(rng, 16, 8192)))
    sinks = rng.choice((0, 1, 4, 64)) if window else 0
    if op in ("write", "read"):
        if rng.random() < 0.4:                                   # single tokens, or a few
            seqs, q = _log_uniform(rng, 1, 96), rng.choice((1, 1, 1, 2, 5, 16))
        else:
            seqs = rng.choice((1, 2, 3, 5))
            q = _log_uniform(rng, 17, 24000 // seqs)
        before = _log_uniform(rng, 1, 4000) - 1
        return _case(None, op, fmt, seqs, q + before, q + rng.randint(0, before), heads, group, dim, page, q_hi=q, q_lo=rng.randint(1, q))
    if op == "shared":
        seqs, prefix, hi = _log_uniform(rng, 2, 96), _log_uniform(rng, 64, 40000), _log_uniform(rng, 1, 1500)
        q = rng.choice((1, 1, 1, 4))
        return _case(None, op, fmt, seqs, hi, rng.randint(1, hi), heads, group, dim, page, q_hi=q, q_lo=1, window=window, sinks=sinks, prefix=prefix)
    weights = rng.choice((0, 0, 1))
    if rng.random() < 0.6:                                       # single tokens, or a few
        seqs = _log_uniform(rng, 1, 64)
        hi = _log_uniform(rng, 16, min(131072, (1 << 22) // (seqs * heads)))
        q = rng.choice((1, 1, 1, 2, 5, 11))
        return _case(None, op, fmt, seqs, hi, rng.randint(0, hi), heads, group, dim, page, q_hi=q, q_lo=rng.randint(1, q), window=window, sinks=sinks,
                     weights=weights)
    seqs = rng.choice((1, 2, 3))
    q, before = _log_uniform(rng, 17, 6000), _log_uniform(rng, 1, 4000) - 1
    most = 5e11 / (4 * dim * heads * group * seqs)               # pairs of a query and a token
    while q * (q + before) > most:
        q, before = q * 3 // 4, before * 3 // 4
    hi = q + before
    lo = rng.randint(1, q)
    return _case(None, op, fmt, seqs, hi, max(lo, hi - rng.randint(0, hi)), heads, group, dim, page, q_hi=q, q_lo=lo, window=window, sinks=sinks, weights=weights)


# ------------------------------------------------------------------------------------------- sizes and inputs

def _spread(hi, lo, n):
    return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _sizes(case):
    """(tokens in the caches, tokens written, read or asked with) of the sequences."""
    return _spread(case["kv_hi"], case["kv_lo"], case["seqs"]), _spread(case["q_hi"], case["q_lo"], case["seqs"])


def _row_bytes(fmt, dim):
    """Bytes of a stored row of K or V, its block scales included."""
    return {"bf16": 2 * dim, "fp8": dim, "e5m2": dim}.get(fmt) or dim // 2 + dim // BLOCK[fmt]


def _seen(case, position):
    """Tokens that a query at a position sees."""
    n = max(0, position + 1)
    if case["window"] and n > case["window"]:
        return case["window"] + min(case["sinks"], n - case["window"])
    return n


def work(case):
    row = 2 * _row_bytes(case["fmt"], case["dim"])               # a token's K and V of one head
    lens, qs = _sizes(case)
    if case["op"] in ("write", "read"):
        wide = 2 * case["dim"] * 2                               # the same in BF16
        return {"bytes": sum(qs) * case["heads"] * (row + (2 if case["op"] == "write" else 1) * wide), "flops": 0}
    pairs = sum(_seen(case, case["prefix"] + n - q + i) for n, q in zip(lens, qs) for i in range(q))
    rows, first_prefix = 0, case["prefix"]
    for n, q in zip(lens, qs):                                   # cached tokens that some query of the sequence sees
        first = max(0, case["prefix"] + n - q - case["window"] + 1) if case["window"] else 0
        first_prefix = min(first_prefix, first)
        if case["prefix"]:
            rows += n - min(n, max(0, first - case["prefix"]))
        else:
            rows += n - max(0, min(n, first) - min(case["sinks"], min(n, first)))
    if case["prefix"]:
        rows += case["prefix"] - max(0, first_prefix - case["sinks"])
    qo = sum(qs) * case["heads"] * case["group"] * (2 * case["dim"] * 2 + 4)
    return {"bytes": rows * case["heads"] * row + qo + (8 * sum(lens) * case["heads"] if case["weights"] else 0),
            "flops": 4 * case["dim"] * case["heads"] * case["group"] * pairs}


def _values(shape, g):
    """K and V [seqs, heads, tokens, dim]: V ~ N(0, 1); K ~ N(0, 1) with four outlier channels per head at ten times that and a slow drift."""
    v, k = torch.randn(shape, generator=g, device="cuda"), torch.randn(shape, generator=g, device="cuda")
    sigma = torch.ones(shape[1], shape[3], device="cuda")
    sigma.scatter_(1, torch.rand(sigma.shape, generator=g, device="cuda").argsort(1)[:, :4], 10.0)
    t = torch.arange(shape[2], device="cuda", dtype=torch.float32)
    return k * sigma.view(1, shape[1], 1, -1) + 0.1 * torch.sin(t / 512.0).view(1, 1, -1, 1), v


def _e2m1(y):
    """Codes of the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, ties to even codes."""
    a = y.abs()
    code = torch.zeros(y.shape, dtype=torch.uint8, device=y.device)
    code += a > TIES[0]
    code += a >= TIES[1]
    code += a > TIES[2]
    code += a >= TIES[3]
    code += a > TIES[4]
    code += a >= TIES[5]
    code += a > TIES[6]
    return code | (torch.signbit(y).to(torch.uint8) << 3)


def _stored(y, fmt):
    """float32 [..., dim], already divided by the scale per sequence and head -> (stored elements, block scales or None)."""
    if fmt == "bf16":
        return y.to(torch.bfloat16).view(torch.int16), None
    if fmt in FP8:
        return y.clamp(-LARGEST[fmt], LARGEST[fmt]).to(FP8[fmt]).view(torch.uint8), None
    blocks = y.unflatten(-1, (-1, BLOCK[fmt]))
    largest = blocks.abs().amax(dim=-1, keepdim=True)
    if fmt == "mx":
        e = torch.frexp(largest).exponent - 3                    # (frexp's mantissa is in 0.5 .. 1)
        e = torch.where(largest > 0, e, torch.full_like(e, -127)).clamp(-127, 127)
        scales = (e + 127).to(torch.uint8)
        blocks = blocks * torch.exp2(-e.to(torch.float32))
    else:
        rounded = (largest / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
        scales, s = rounded.view(torch.uint8), rounded.to(torch.float32)
        blocks = torch.where(s > 0, blocks / s, torch.zeros_like(blocks))
    code = _e2m1(blocks).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), scales.squeeze(-1)


def _of_stored(bits, scales, fmt):
    """Stored elements (and their block scales) -> float32."""
    if fmt == "bf16":
        return bits.view(torch.bfloat16).to(torch.float32)
    if fmt in FP8:
        return bits.view(FP8[fmt]).to(torch.float32)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=bits.device)
    code = torch.stack([bits & 15, bits >> 4], dim=-1).flatten(-2)
    x = grid[(code & 7).to(torch.int64)]
    x = torch.where(code >= 8, -x, x).unflatten(-1, (-1, BLOCK[fmt]))
    s = torch.exp2(scales.to(torch.float32) - 127.0) if fmt == "mx" else scales.view(torch.float8_e4m3fn).to(torch.float32)
    if fmt == "mx":
        s = torch.where(scales == 255, torch.full_like(s, math.nan), s)
    return (x * s.unsqueeze(-1)).flatten(-2)


def _nothing(fmt, shape, dim):
    """Pools of pages that hold NaN: elements, block scales or None."""
    if fmt == "bf16":
        return torch.full(shape + (dim,), 0x7FFF, dtype=torch.int16, device="cuda"), None
    if fmt in FP8:
        return torch.full(shape + (dim,), 0x7F, dtype=torch.uint8, device="cuda"), None
    return (torch.full(shape + (dim // 2,), 0xFF, dtype=torch.uint8, device="cuda"),
            torch.full(shape + (dim // BLOCK[fmt],), 255 if fmt == "mx" else 127, dtype=torch.uint8, device="cuda"))


def _cache(case, lens, g, empty=False):
    """A paged cache: pools of pages as stored, their block scales, the table, the lengths, the scales per sequence and head.  Under
    "k_values" and "v_values" what it is made of.  empty: nothing has been written to it."""
    page, fmt, seqs, dim, heads = case["page"], case["fmt"], len(lens), case["dim"], case["heads"]
    pages = max(1, -(-max(lens) // page))
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    used = seqs * heads * pages
    order = torch.randperm(used + 5, generator=g, device="cuda")[:used]
    c = {"table": order.view(seqs, heads, pages).to(torch.int32), "lengths": lengths}
    inside = (torch.arange(pages * page, device="cuda") < lengths.view(-1, 1)).view(seqs, 1, pages, page).expand(-1, heads, -1, -1).reshape(used, page)
    for name, x in zip("kv", _values((seqs, heads, pages * page, dim), g)):
        scale = x.abs().amax(dim=(2, 3)) / LARGEST[fmt] if fmt in LARGEST else None
        c[name + "_scale"] = scale
        c[name], c[name + "_blocks"] = _nothing(fmt, (used + 5, page), dim)
        if empty:
            c[name + "_values"] = x
            continue
        bits, blocks = _stored(x if scale is None else x / scale[:, :, None, None], fmt)
        where = order[:, None].expand(-1, page)[inside] * page + torch.arange(page, device="cuda").expand(used, -1)[inside]
        c[name].view(-1, c[name].shape[2])[where] = bits.view(used, page, -1)[inside]
        if blocks is not None:
            c[name + "_blocks"].view(-1, blocks.shape[-1])[where] = blocks.view(used, page, -1)[inside]
    return c


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed & 0x7FFFFFFF)
    lens, qs = _sizes(case)
    s = {"case": case, "cache": _cache(case, lens, g, empty=case["op"] == "write"), "lens": lens, "qs": qs}
    n, heads, dim = sum(qs), case["heads"], case["dim"]
    # where each of the tokens belongs: what the plain form goes by, and what the library is told
    s["q_start"] = torch.tensor([sum(qs[:i]) for i in range(len(qs) + 1)], dtype=torch.int32, device="cuda")
    s["q_lens"] = torch.tensor(qs, dtype=torch.int64, device="cuda")
    s["token_seq"] = torch.repeat_interleave(torch.arange(len(qs), device="cuda"), s["q_lens"])
    s["token_at"] = torch.arange(n, device="cuda") - s["q_start"].to(torch.int64)[s["token_seq"]]
    if case["op"] == "write":
        # keys and values as a projection leaves them: a token's query, key and value heads side by side
        at = (s["cache"]["lengths"].to(torch.int64) - s["q_lens"])[s["token_seq"]] + s["token_at"]
        rows = torch.empty((n, (case["group"] + 2) * heads, dim), dtype=torch.bfloat16, device="cuda")
        rows.normal_(generator=g)
        s["k"], s["v"] = rows[:, case["group"] * heads:-heads], rows[:, -heads:]
        for name in "kv":
            s[name].copy_(s["cache"].pop(name + "_values")[s["token_seq"], :, at])
        return s
    if case["op"] == "read":
        return s
    s["q"] = torch.randn((n, heads * case["group"], dim), generator=g, device="cuda").to(torch.bfloat16)
    if case["op"] == "shared":
        s["prefix"] = _cache(case, [case["prefix"]], g)
    if case["weights"]:
        s["weights"] = torch.rand((case["seqs"], heads, s["cache"]["table"].shape[2] * case["page"]), generator=g, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["weights"]:
        s["weights_out"] = torch.zeros_like(s["weights"])
    if own:
        from paper_2508_19263_amd import zc
        fmt = {"bf16": zc.FMT_BF16, "fp8": zc.FMT_FP8_E4M3, "e5m2": zc.FMT_FP8_E5M2, "mx": zc.FMT_FP4_E2M1_MX, "nv": zc.FMT_FP4_E2M1_NV}[case["fmt"]]
        for name in ("cache", "prefix"):
            if name in s:
                c = s[name]
                s["zc_" + name] = zc.PagedCache(c["k"], c["v"], c["table"], c["lengths"], fmt, c["k_scale"], c["v_scale"], c["k_blocks"], c["v_blocks"])
    return s


# --------------------------------------------------------------------------------------------------- the calls

def run(s):
    if own:
        return _run_own(s)
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend, "shared": _plain_attend}[s["case"]["op"]](s)


def _run_own(s):
    from paper_2508_19263_amd import zc
    case = s["case"]
    several = case["q_hi"] > 1 or case["q_lo"] < 1
    start = s["q_start"] if several else None
    if case["op"] in ("write", "read"):
        if case["op"] == "write":
            zc.write_kv(s["k"], s["v"], s["zc_cache"], q_start=start)
        k, v = zc.read_kv(s["zc_cache"], q_start=start, n_tokens=sum(s["qs"]))
        return {"k": k, "v": v}
    more = dict(window=case["window"], sinks=case["sinks"], max_kv_len=case["kv_hi"])
    if several:
        more.update(q_start=start, max_q_len=case["q_hi"])
    if case["op"] == "shared":
        out, lse = zc.attend_shared(s["q"], s["zc_prefix"], s["zc_cache"], max_prefix_len=case["prefix"], **more)
        return {"out": out, "lse": lse}
    if case["weights"]:
        out, lse = zc.attend(s["q"], s["zc_cache"], weights=s["weights"], weights_out=s["weights_out"], **more)
        return {"out": out, "lse": lse, "weights": s["weights_out"]}
    out, lse = zc.attend(s["q"], s["zc_cache"], **more)
    return {"out": out, "lse": lse}


def _rows_of_tokens(s):
    """[tokens, heads]: the row of the pools that each of the tokens has in its head's pages."""
    c, page = s["cache"], s["case"]["page"]
    at = (c["lengths"].to(torch.int64) - s["q_lens"])[s["token_seq"]] + s["token_at"]
    return c["table"].to(torch.int64)[s["token_seq"], :, at // page] * page + (at % page).unsqueeze(1)


def _plain_write(s):
    c, fmt = s["cache"], s["case"]["fmt"]
    rows = _rows_of_tokens(s).reshape(-1)
    for name in "kv":
        x = s[name].to(torch.float32)
        if c[name + "_scale"] is not None:
            x = x / c[name + "_scale"][s["token_seq"]].unsqueeze(-1)
        bits, blocks = _stored(x, fmt)
        c[name].view(-1, bits.shape[-1])[rows] = bits.flatten(0, 1)
        if blocks is not None:
            c[name + "_blocks"].view(-1, blocks.shape[-1])[rows] = blocks.flatten(0, 1)
    return _plain_read(s)


def _plain_read(s):
    c, fmt, res = s["cache"], s["case"]["fmt"], {}
    rows = _rows_of_tokens(s)
    for name in "kv":
        blocks = c[name + "_blocks"]
        x = _of_stored(c[name].view(-1, c[name].shape[2])[rows], None if blocks is None else blocks.view(-1, blocks.shape[2])[rows], fmt)
        if c[name + "_scale"] is not None:
            x = x * c[name + "_scale"][s["token_seq"]].unsqueeze(-1)
        res[name] = x.to(torch.bfloat16)
    return res


def _dense(c, name, fmt):
    """[seqs, heads, tokens, dim] in float32, zero behind a sequence's end."""
    table, blocks = c["table"].to(torch.int64), c[name + "_blocks"]
    x = _of_stored(c[name][table], None if blocks is None else blocks[table], fmt).flatten(2, 3)
    inside = torch.arange(x.shape[2], device=x.device) < c["lengths"].view(-1, 1)
    x = torch.where(inside[:, None, :, None], x, torch.zeros_like(x))
    return x if c[name + "_scale"] is None else x * c[name + "_scale"][:, :, None, None]


def _visible(position, tokens, first, length, window, sinks):
    """[seqs, queries, tokens]: token j, at position first + j, is there and seen from `position`."""
    at = torch.arange(tokens, device=position.device)
    key, position = at + first, position.unsqueeze(-1)
    seen = (key <= position) & (at < length.view(-1, 1, 1))
    return seen & ((key > position - window) | (key < sinks)) if window else seen


def _plain_attend(s):
    case, fmt = s["case"], s["case"]["fmt"]
    S, H, G, D, Q = case["seqs"], case["heads"], case["group"], case["dim"], case["q_hi"]
    window, sinks, P = case["window"], case["sinks"], case["prefix"]
    length = s["cache"]["lengths"].to(torch.int64)
    q = torch.zeros((S, Q, H * G, D), device="cuda")
    q[s["token_seq"], s["token_at"]] = s["q"].to(torch.float32)
    q = q.view(S, Q, H, G, D).permute(0, 2, 1, 3, 4).reshape(S, H, Q * G, D) / math.sqrt(D)
    position = (P + length - s["q_lens"]).unsqueeze(1) + torch.arange(Q, device="cuda")
    k, v = _dense(s["cache"], "k", fmt), _dense(s["cache"], "v", fmt)
    tokens = k.shape[2]
    logits = torch.matmul(q, k.transpose(2, 3)).view(S, H, Q, G, tokens)
    seen = _visible(position, tokens, P, length, window, sinks)
    if P:
        pk, pv = _dense(s["prefix"], "k", fmt)[0], _dense(s["prefix"], "v", fmt)[0]
        of_prefix = torch.matmul(q.transpose(0, 1).reshape(H, S * Q * G, D), pk.transpose(1, 2)).view(H, S, Q, G, -1).transpose(0, 1)
        logits = torch.cat([of_prefix, logits], dim=-1)
        seen = torch.cat([_visible(position, pk.shape[1], 0, s["prefix"]["lengths"], window, sinks), seen], dim=-1)
    logits = logits.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    m = logits.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = logits.sub_(m).exp_()
    total = p.sum(dim=-1, keepdim=True)
    lse = (m + torch.log(total)).squeeze(-1)
    p = p.div_(torch.where(total == 0, torch.ones_like(total), total))
    if P:
        of_prefix = p[..., :-tokens].transpose(0, 1).reshape(H, S * Q * G, -1)
        out = torch.matmul(of_prefix, pv).view(H, S, Q * G, D).transpose(0, 1) + torch.matmul(p[..., -tokens:].reshape(S, H, Q * G, -1), v)
    else:
        out = torch.matmul(p.view(S, H, Q * G, tokens), v)
    out = out.view(S, H, Q, G, D).permute(0, 2, 1, 3, 4).reshape(S, Q, H * G, D)
    res = {"out": out[s["token_seq"], s["token_at"]].to(torch.bfloat16),
           "lse": lse.permute(0, 2, 1, 3).reshape(S, Q, H * G)[s["token_seq"], s["token_at"]]}
    if case["weights"]:
        asked = (torch.arange(Q, device="cuda") < s["q_lens"].view(-1, 1)).to(torch.float32)
        given = torch.matmul(asked.repeat_interleave(G, dim=1).view(S, 1, 1, Q * G), p.view(S, H, Q * G, tokens)).squeeze(2)
        inside = (torch.arange(tokens, device="cuda") < length.view(-1, 1)).unsqueeze(1)
        s["weights_out"].copy_(torch.where(inside, s["weights"] + given, torch.zeros_like(given)))
        res["weights"] = s["weights_out"]
    return res


# ------------------------------------------------------------------------------------------------ in 64 bits

FLOATS = {"fp8": (3, -6, 448.0), "e5m2": (2, -14, 57344.0), "e2m1": (1, 0, 6.0)}     # bits of the mantissa, least exponent, largest number


def _nearest(y, kind):
    """The numbers of a small float type next to y."""
    mantissa, least, largest = FLOATS[kind]
    step = torch.exp2((torch.frexp(y).exponent - 1).clamp(min=least).to(torch.float64) - mantissa)
    return (torch.round(y / step) * step).clamp(-largest, largest)


def _kept(x, scale, fmt):
    """float64 [rows, dim] of one head: what is left of it when it has been quantised and read back."""
    y = x if scale is None else x / scale
    if fmt in FP8:
        y = _nearest(y, fmt)
    elif fmt in BLOCK:
        y = y.view(y.shape[0], -1, BLOCK[fmt])
        top = y.abs().amax(dim=2, keepdim=True)
        if fmt == "mx":
            s = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top)))) - 2)
        else:
            s = _nearest(top / 6, "fp8")
        y = (_nearest(torch.where(s > 0, y / s, torch.zeros_like(y)), "e2m1") * s).view(x.shape)
    return y if scale is None else y * scale


def exact(case, seed):
    s = _inputs(case, seed)
    lens, qs, page, D, G, fmt = s["lens"], s["qs"], case["page"], case["dim"], case["group"], case["fmt"]

    def scale_of(c, name, seq, head):
        return None if c[name + "_scale"] is None else c[name + "_scale"][seq, head].to(torch.float64)

    def rows(c, name, seq, head, n):
        """The first n tokens' rows of one head in 64 bits."""
        if not n:
            return torch.zeros((0, D), dtype=torch.float64, device="cuda")
        pages = c["table"][seq, head, :-(-n // page)].to(torch.int64)
        bits = c[name][pages].flatten(0, 1)[:n]
        if fmt in BLOCK:
            x = torch.zeros((n, D), dtype=torch.float64, device="cuda")
            for half in range(2):
                code = (bits >> 4 * half & 15).to(torch.float64)
                e, m = torch.floor((code % 8) / 2), code % 2
                x[:, half::2] = torch.where(code >= 8, -1.0, 1.0) * torch.where(e > 0, torch.exp2(e - 1) * (1 + m / 2), m / 2)
            b = c[name + "_blocks"][pages].flatten(0, 1)[:n]
            b = torch.exp2(b.to(torch.float64) - 127) if fmt == "mx" else b.view(torch.float8_e4m3fn).to(torch.float64)
            x = x * b.repeat_interleave(BLOCK[fmt], dim=1)
        else:
            x = bits.view(FP8.get(fmt, torch.bfloat16)).to(torch.float64)
        scale = scale_of(c, name, seq, head)
        return x if scale is None else x * scale

    total, P = sum(qs), case["prefix"]
    if case["op"] in ("write", "read"):
        res = {name: torch.zeros((total, case["heads"], D), dtype=torch.float64, device="cuda") for name in "kv"}
        for i, (n, nq) in enumerate(zip(lens, qs)):
            first = sum(qs[:i])
            for h in range(case["heads"]):
                for name in "kv":
                    if case["op"] == "write":
                        res[name][first:first + nq, h] = _kept(s[name][first:first + nq, h].to(torch.float64), scale_of(s["cache"], name, i, h), fmt)
                    else:
                        res[name][first:first + nq, h] = rows(s["cache"], name, i, h, n)[n - nq:]
        return res

    out = torch.zeros((total, case["heads"] * G, D), dtype=torch.float64, device="cuda")
    lse = torch.full((total, case["heads"] * G), -math.inf, dtype=torch.float64, device="cuda")
    weights = torch.zeros(s["weights"].shape, dtype=torch.float64, device="cuda") if case["weights"] else None
    for i, (n, nq) in enumerate(zip(lens, qs)):
        first = sum(qs[:i])
        if weights is not None:
            weights[i, :, :n] = s["weights"][i, :, :n].to(torch.float64)
        if P + n == 0:
            continue
        position = (P + n - nq + torch.arange(nq, device="cuda")).view(-1, 1)
        key = torch.arange(P + n, device="cuda")
        hidden = key > position
        if case["window"]:
            hidden |= (key <= position - case["window"]) & (key >= case["sinks"])
        for h in range(case["heads"]):
            k, v = rows(s["cache"], "k", i, h, n), rows(s["cache"], "v", i, h, n)
            if P:
                k, v = torch.cat([rows(s["prefix"], "k", 0, h, P), k]), torch.cat([rows(s["prefix"], "v", 0, h, P), v])
            for g in range(G):
                x = s["q"][first:first + nq, h * G + g].to(torch.float64) @ k.t() * D ** -0.5
                x.masked_fill_(hidden, -math.inf)
                z = torch.logsumexp(x, dim=1)
                p = torch.exp(x - torch.where(z == -math.inf, torch.zeros_like(z), z).unsqueeze(1))
                out[first:first + nq, h * G + g], lse[first:first + nq, h * G + g] = p @ v, z
                if weights is not None:
                    weights[i, h, :n] += p.sum(dim=0)
    return {"out": out, "lse": lse} if weights is None else {"out": out, "lse": lse, "weights": weights}
