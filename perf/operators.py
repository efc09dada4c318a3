"""The operators over K/V pages, as measurable cases.

A page is `page` tokens of one K/V head of one sequence, [page][dim] elements; a table gives the page of every stretch of
`page` tokens.  Pages of a pool lie in random order, tokens behind a sequence's end and pages that no table names hold
whatever was there before (NaN bytes here).  A case is a dict of plain values:
  op       "attend" (attention with a sliding window and sinks), "shared" (a batch that shares a prefix), "evict"
  fmt      element format of the pages: "bf16", "fp8" (E4M3) or "e5m2", the latter two with a float scale per sequence and head
  seqs, heads, group, dim, page   sequences, K/V heads, query heads per K/V head, head dimension, tokens per page
  kv_hi, kv_lo   lengths of the sequences' own caches, spread evenly from the one to the other
  q_hi, q_lo     query tokens per sequence, spread likewise
  window, sinks  0: every earlier token is visible
  prefix   tokens of the shared prefix
  weights  1: the attention weight of every cached token is added up too
  keep, recent   tokens that eviction leaves, and how many of the newest are among them whatever their weight

Query i of a sequence of n query tokens is at position len - n + i.  Where `own` is false the operators are computed from
elementary torch operations in 32 bits, else by the library's kernels.
"""
import math

import torch

own = False

TORCH_TYPE = {"bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"fp8": 448.0, "e5m2": 57344.0}
NAN_BYTE = 0x7F                                                  # a NaN in both FP8 formats; twice that, one in BF16


def _case(name, op, fmt, seqs, kv_hi, kv_lo, heads=8, group=4, dim=128, page=16, q_hi=1, q_lo=1, window=0, sinks=0, prefix=0, weights=0, keep=0,
          recent=0):
    c = dict(op=op, fmt=fmt, seqs=seqs, heads=heads, group=group, dim=dim, page=page, kv_hi=kv_hi, kv_lo=kv_lo, q_hi=q_hi, q_lo=q_lo,
             window=window, sinks=sinks, prefix=prefix, weights=weights, keep=keep, recent=recent)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the next token of one conversation: the smallest call, latency alone
        _case("decode_one", "attend", "fp8", 1, 1000, 1000, window=512, sinks=4),
        # the next tokens of the batch that fills the FP8 cache of workloads.fp8_kv_pair
        _case("decode_batch", "attend", "fp8", 4, 8192, 8192),
        # a server's batch at all stages, an empty slot among them, with a window that has left the first pages of most behind
        _case("decode_window_ragged", "attend", "bf16", 32, 30011, 0, group=8, window=4096, sinks=16),
        # five drafted tokens per sequence to be checked at once, small heads
        _case("decode_draft", "attend", "e5m2", 6, 7919, 3001, group=7, dim=64, q_hi=5, q_lo=5, window=2048, sinks=64),
        # a piece of two long prompts over what is cached of them already
        _case("prefill_chunk", "attend", "fp8", 2, 9001, 8191, q_hi=1024, q_lo=511, window=4096, sinks=4),
        # two whole prompts: the largest call
        _case("prefill_long", "attend", "bf16", 2, 8192, 7001, q_hi=8192, q_lo=7001, window=4096, sinks=16),
        # a few answers to one short question
        _case("shared_few", "shared", "bf16", 5, 200, 1, prefix=1531),
        # many answers under one long document
        _case("shared_many", "shared", "fp8", 64, 777, 16, prefix=32768),
        # a decoding step that keeps account of every token's weight
        _case("weights_decode", "attend", "fp8", 4, 8192, 8192, weights=1),
        # the same over a prompt
        _case("weights_prompt", "attend", "bf16", 1, 4099, 4099, q_hi=4099, q_lo=4099, weights=1),
        # half of the FP8 cache goes
        _case("evict_half", "evict", "fp8", 4, 8192, 8192, sinks=4, keep=4096, recent=1024),
        # a batch of long conversations cut down to one length
        _case("evict_long", "evict", "bf16", 16, 65536, 20011, sinks=16, keep=8191, recent=500),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(("attend", "attend", "attend", "shared", "evict"))
    fmt = rng.choice(("fp8", "bf16", "e5m2"))
    heads, group, dim, page = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 3, 4, 5, 7, 8)), rng.choice((128, 128, 64)), rng.choice((16, 16, 32, 64))
    window = rng.choice((0, 0, _log_uniform(rng, 16, 8192)))
    sinks = rng.choice((0, 1, 4, 64)) if window else 0
    if op == "evict":
        seqs = _log_uniform(rng, 1, 32)
        hi = _log_uniform(rng, 64, min(65536, (1 << 23) // (seqs * heads)))
        keep = max(8, int(hi * rng.uniform(0.1, 0.9)))
        return _case(None, op, fmt, seqs, hi, int(hi * rng.uniform(0.05, 1.0)), heads, group, dim, page, sinks=rng.choice((0, 4)), keep=keep,
                     recent=int((keep - 4) * rng.choice((0.0, 0.25, 0.5))))
    if op == "shared":
        seqs, prefix, hi = _log_uniform(rng, 2, 96), _log_uniform(rng, 64, 40000), _log_uniform(rng, 1, 1500)
        q = rng.choice((1, 1, 1, 4))
        return _case(None, op, fmt, seqs, hi, rng.randint(1, hi), heads, group, dim, page, q_hi=q, q_lo=1, window=window, sinks=sinks, prefix=prefix)
    weights = rng.choice((0, 0, 1))
    if rng.random() < 0.6:                                      # single tokens, or a few
        seqs = _log_uniform(rng, 1, 64)
        hi = _log_uniform(rng, 16, min(131072, (1 << 22) // (seqs * heads)))
        q = rng.choice((1, 1, 1, 2, 5, 11))
        return _case(None, op, fmt, seqs, hi, rng.randint(0, hi), heads, group, dim, page, q_hi=q, q_lo=rng.randint(1, q), window=window, sinks=sinks,
                     weights=weights)
    seqs = rng.choice((1, 2, 3))
    q, before = _log_uniform(rng, 17, 6000), _log_uniform(rng, 1, 4000) - 1
    most = 7e11 / (4 * dim * heads * group * seqs)               # pairs of a query and a token
    while q * (q + before) > most:
        q, before = q * 3 // 4, before * 3 // 4
    hi = q + before
    lo = rng.randint(1, q)
    return _case(None, op, fmt, seqs, hi, max(lo, hi - rng.randint(0, hi)), heads, group, dim, page, q_hi=q, q_lo=lo, window=window, sinks=sinks, weights=weights)


# ------------------------------------------------------------------------------------------- sizes and inputs

def _spread(hi, lo, n):
    return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _sizes(case):
    """(tokens in the caches, query tokens) of the sequences."""
    return _spread(case["kv_hi"], case["kv_lo"], case["seqs"]), _spread(case["q_hi"], case["q_lo"], case["seqs"])


def _seen(case, position):
    """Tokens that a query at a position sees."""
    n = max(0, position + 1)
    if case["window"] and n > case["window"]:
        return case["window"] + min(case["sinks"], n - case["window"])
    return n


def work(case):
    es = 2 if case["fmt"] == "bf16" else 1
    row = 2 * case["dim"] * es                                   # a token's K and V of one head
    lens, qs = _sizes(case)
    if case["op"] == "evict":
        kept = sum(min(n, case["keep"]) for n in lens)
        return {"bytes": case["heads"] * (4 * sum(lens) + kept * (2 * row + 8)), "flops": 0}
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


def _values(case, seqs, tokens, g):
    """K and V of `seqs` caches as float32 [seqs, heads, tokens, dim]: V ~ N(0, 1); K ~ N(0, 1) with four outlier channels per
    head at ten times that and a slow drift."""
    shape = (seqs, case["heads"], tokens, case["dim"])
    v = torch.randn(shape, generator=g, device="cuda")
    k = torch.randn(shape, generator=g, device="cuda")
    sigma = torch.ones(case["heads"], case["dim"], device="cuda")
    sigma.scatter_(1, torch.rand(sigma.shape, generator=g, device="cuda").argsort(1)[:, :4], 10.0)
    t = torch.arange(tokens, device="cuda", dtype=torch.float32)
    return k * sigma.view(1, case["heads"], 1, -1) + 0.1 * torch.sin(t / 512.0).view(1, 1, tokens, 1), v


def _cache(case, lens, g):
    """A paged cache: pools of pages as stored, the table, the lengths, the scales (None for BF16)."""
    page, fmt, seqs = case["page"], case["fmt"], len(lens)
    pages = max(1, -(-max(lens) // page))
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    used = seqs * case["heads"] * pages
    order = torch.randperm(used + 5, generator=g, device="cuda")[:used]
    c = {"table": order.view(seqs, case["heads"], pages).to(torch.int32), "lengths": lengths}
    inside = (torch.arange(pages * page, device="cuda") < lengths.view(-1, 1)).view(seqs, 1, -1, 1)
    for name, x in zip("kv", _values(case, seqs, pages * page, g)):
        scale = None
        if fmt != "bf16":
            scale = x.abs().amax(dim=(2, 3)) / LARGEST[fmt]
            x = x / scale[:, :, None, None]
        bits = x.to(TORCH_TYPE[fmt]).view(torch.int16 if fmt == "bf16" else torch.uint8)
        junk = NAN_BYTE * 257 if fmt == "bf16" else NAN_BYTE
        bits = torch.where(inside, bits, torch.full_like(bits, junk))
        pool = torch.full((used + 5, page, case["dim"]), junk, dtype=bits.dtype, device="cuda")
        pool[order] = bits.view(used, page, case["dim"])
        c[name], c[name + "_scale"] = pool, scale
    return c


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed & 0x7FFFFFFF)
    lens, qs = _sizes(case)
    s = {"case": case, "cache": _cache(case, lens, g), "lens": lens, "qs": qs}
    capacity = s["cache"]["table"].shape[2] * case["page"]
    if case["op"] == "evict":
        # what rows of softmaxes add up to: a few heavy tokens, many light ones, and a fifth that no query has looked at
        w = torch.rand((case["seqs"], case["heads"], capacity), generator=g, device="cuda").pow(-0.5) - 1
        s["weights"] = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.2, torch.zeros_like(w), w)
        return s
    n = sum(qs)
    s["q"] = torch.randn((n, case["heads"] * case["group"], case["dim"]), generator=g, device="cuda").to(torch.bfloat16)
    if case["op"] == "shared":
        s["prefix"] = _cache(case, [case["prefix"]], g)
    if case["weights"]:
        s["weights"] = torch.rand((case["seqs"], case["heads"], capacity), generator=g, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    lens, qs, dev = s["lens"], s["qs"], "cuda"
    if case["op"] == "evict":
        pages = -(-min(case["keep"], max(lens)) // case["page"])
        used = case["seqs"] * case["heads"] * pages
        into = {"table": torch.arange(used, dtype=torch.int32, device=dev).view(case["seqs"], case["heads"], pages),
                "lengths": torch.zeros(case["seqs"], dtype=torch.int32, device=dev)}
        for name in "kv":
            into[name] = torch.zeros((used, case["page"], case["dim"]), dtype=s["cache"][name].dtype, device=dev)
            into[name + "_scale"] = s["cache"][name + "_scale"]   # they go with the sequence and head
        s["into"], s["into_weights"] = into, torch.zeros((case["seqs"], case["heads"], pages * case["page"]), device=dev)
    else:
        # where each query token belongs: what the plain form pads by, and what the library is told
        s["q_start"] = torch.tensor([sum(qs[:i]) for i in range(len(qs) + 1)], dtype=torch.int32, device=dev)
        s["q_lens"] = torch.tensor(qs, dtype=torch.int64, device=dev)
        s["token_seq"] = torch.repeat_interleave(torch.arange(len(qs), device=dev), s["q_lens"])
        s["token_at"] = torch.arange(sum(qs), device=dev) - s["q_start"].to(torch.int64)[s["token_seq"]]
        if case["weights"]:
            s["weights_out"] = torch.zeros_like(s["weights"])
    if own:
        from paper_2508_19263_amd import zc
        fmt = {"bf16": zc.FMT_BF16, "fp8": zc.FMT_FP8_E4M3, "e5m2": zc.FMT_FP8_E5M2}[case["fmt"]]
        for name in ("cache", "prefix", "into"):
            if name in s:
                c = s[name]
                s["zc_" + name] = zc.PagedCache(c["k"], c["v"], c["table"], c["lengths"], fmt, c["k_scale"], c["v_scale"])
    return s


# --------------------------------------------------------------------------------------------------- the calls

def run(s):
    if own:
        return _run_own(s)
    return {"attend": _plain_attend, "shared": _plain_attend, "evict": _plain_evict}[s["case"]["op"]](s)


def _run_own(s):
    from paper_2508_19263_amd import zc
    case = s["case"]
    if case["op"] == "evict":
        kept = zc.evict(s["zc_cache"], s["weights"], case["keep"], s["zc_into"], s["into_weights"], sinks=case["sinks"], recent=case["recent"])
        return _evicted(s, kept)
    more = dict(window=case["window"], sinks=case["sinks"], max_kv_len=case["kv_hi"])
    if case["q_hi"] > 1 or case["q_lo"] < 1:
        more.update(q_start=s["q_start"], max_q_len=case["q_hi"])
    if case["op"] == "shared":
        out, lse = zc.attend_shared(s["q"], s["zc_prefix"], s["zc_cache"], max_prefix_len=case["prefix"], **more)
        return {"out": out, "lse": lse}
    if case["weights"]:
        out, lse = zc.attend(s["q"], s["zc_cache"], weights=s["weights"], weights_out=s["weights_out"], **more)
        return {"out": out, "lse": lse, "weights": s["weights_out"]}
    out, lse = zc.attend(s["q"], s["zc_cache"], **more)
    return {"out": out, "lse": lse}


def _evicted(s, kept):
    into, t = s["into"], TORCH_TYPE[s["case"]["fmt"]]
    return {"kept": kept, "lengths": into["lengths"], "k": into["k"].view(t), "v": into["v"].view(t), "weights": s["into_weights"]}


def _dense(c, name, fmt):
    """[seqs, heads, tokens, dim] in float32, zero behind a sequence's end."""
    pool, table = c[name], c["table"]
    x = pool[table.to(torch.int64)].view(TORCH_TYPE[fmt]).to(torch.float32).flatten(2, 3)
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


def _plain_evict(s):
    case, c, into = s["case"], s["cache"], s["into"]
    length = c["lengths"].to(torch.int64).view(-1, 1, 1)
    tokens = s["weights"].shape[2]
    at = torch.arange(tokens, device="cuda")
    kept_anyway = (at < case["sinks"]) | (at >= length - case["recent"])
    key = torch.where(kept_anyway, torch.full_like(s["weights"], math.inf), s["weights"])
    key = torch.where(at < length, key, torch.full_like(key, -math.inf))
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :case["keep"]]
    count = torch.clamp(length, max=case["keep"])
    valid = torch.arange(order.shape[2], device="cuda") < count
    kept = torch.where(valid, order, torch.full_like(order, tokens)).sort(dim=-1).values
    source = kept.clamp(max=tokens - 1)
    page, D = case["page"], case["dim"]
    slots = into["table"].shape[2] * page
    room = (0, slots - min(slots, source.shape[2]))
    source = torch.nn.functional.pad(source[..., :slots], room)
    live = torch.nn.functional.pad(valid[..., :slots].expand(source.shape[0], source.shape[1], -1), room)
    from_page = torch.gather(c["table"].to(torch.int64), 2, source // page)
    to_page = into["table"].to(torch.int64).reshape(-1)
    for name in "kv":
        rows = c[name].view(-1, D)[from_page * page + source % page]
        rows = torch.where(live.unsqueeze(-1), rows, torch.zeros_like(rows))
        into[name][to_page] = rows.view(-1, page, D)
    s["into_weights"].copy_(torch.where(live, torch.gather(s["weights"], 2, source), torch.zeros((), device="cuda")))
    into["lengths"].copy_(count.view(-1))
    kept = torch.where(valid, kept, torch.full_like(kept, -1)).to(torch.int32)
    return _evicted(s, torch.nn.functional.pad(kept, (0, case["keep"] - kept.shape[2]), value=-1))


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    lens, qs, page, D, G = s["lens"], s["qs"], case["page"], case["dim"], case["group"]

    def rows(c, name, seq, head, n):
        """The first n tokens' rows of one head in 64 bits."""
        pages = c["table"][seq, head, :-(-n // page)].tolist()
        if not n:
            return torch.zeros((0, D), dtype=torch.float64, device="cuda")
        x = c[name][torch.tensor(pages, device="cuda")].view(TORCH_TYPE[case["fmt"]]).to(torch.float64).reshape(-1, D)[:n]
        return x if c[name + "_scale"] is None else x * c[name + "_scale"][seq, head].to(torch.float64)

    if case["op"] == "evict":
        slots = -(-min(case["keep"], max(lens)) // page) * page
        shape = (case["seqs"], case["heads"], slots)
        kept = torch.full((case["seqs"], case["heads"], case["keep"]), -1, dtype=torch.int32, device="cuda")
        k = torch.zeros(shape + (D,), dtype=torch.float64, device="cuda")
        v, w = torch.zeros_like(k), torch.zeros(shape, dtype=torch.float64, device="cuda")
        for i, n in enumerate(lens):
            for h in range(case["heads"]):
                x = s["weights"][i, h, :n].to(torch.float64)
                at = torch.arange(n, device="cuda")
                if n > case["keep"]:
                    middle = at[case["sinks"]:n - case["recent"]]
                    best = middle[torch.argsort(-x[middle], stable=True)[:case["keep"] - case["sinks"] - case["recent"]]]
                    at = torch.cat([at[:case["sinks"]], best.sort().values, at[n - case["recent"]:]])
                m = at.numel()
                kept[i, h, :m], w[i, h, :m] = at.to(torch.int32), x[at]
                plain = dict(s["cache"], k_scale=None, v_scale=None)     # elements are moved as they are stored
                k[i, h, :m], v[i, h, :m] = rows(plain, "k", i, h, n)[at], rows(plain, "v", i, h, n)[at]
        lengths = torch.tensor([min(n, case["keep"]) for n in lens], dtype=torch.int32, device="cuda")
        return {"kept": kept, "lengths": lengths, "k": k.view(-1, page, D), "v": v.view(-1, page, D), "weights": w}

    total, P = sum(qs), case["prefix"]
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
