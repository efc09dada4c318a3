"""What the calls over K/V pages refuse, before anything is queued (no GPU needed: the addresses are never followed)."""
import ctypes as C

import pytest
import torch

from paper_2508_19263_amd import zc

SOME = 0x10000                                                   # an aligned address


def cache(**change):
    c = zc.KvCache()
    c.struct_size, c.format = C.sizeof(zc.KvCache), zc.FMT_FP8_E4M3
    c.n_seqs, c.n_heads, c.head_dim, c.page_tokens, c.table_pages, c.n_pages = 3, 2, 128, 16, 10, 100
    c.d_k_pages = c.d_v_pages = c.d_table = SOME
    c.d_lengths = SOME
    for name, v in change.items():
        setattr(c, name, v)
    return c


def args(**change):
    a = zc.AttendArgs()
    a.struct_size = C.sizeof(zc.AttendArgs)
    a.n_tokens, a.n_q_heads, a.max_q_len, a.scale = 3, 8, 1, 0.1
    a.d_q = a.d_out = a.d_lse = SOME
    a.q_token_stride = a.out_token_stride = 1024
    a.q_head_stride = a.out_head_stride = 128
    for name, v in change.items():
        setattr(a, name, v)
    return a


def attend(a, c, ws=SOME, ws_bytes=0):
    return zc.lib().zc_attend(C.byref(a) if a is not None else None, C.byref(c) if c is not None else None, ws, ws_bytes, None)


def shared(a, p, c, ws=SOME, ws_bytes=0):
    return zc.lib().zc_attend_shared(C.byref(a), C.byref(p) if p is not None else None, C.byref(c), ws, ws_bytes, None)


def evict(f, t, keep=20, sinks=0, recent=0, w=SOME, w_to=None, kept=SOME):
    return zc.lib().zc_evict(C.byref(f), w, keep, sinks, recent, C.byref(t), w_to, kept, None)


BAD_CACHE = [(dict(struct_size=8), zc.ERR_UNSUPPORTED), (dict(format=zc.FMT_FP4_E2M1_MX), zc.ERR_UNSUPPORTED), (dict(format=zc.FMT_FP8_E4M3_BYTES), zc.ERR_UNSUPPORTED),
             (dict(format=0), zc.ERR_UNSUPPORTED), (dict(head_dim=96), zc.ERR_UNSUPPORTED), (dict(head_dim=0), zc.ERR_UNSUPPORTED),
             (dict(page_tokens=8), zc.ERR_INVALID_ARG), (dict(page_tokens=24), zc.ERR_INVALID_ARG), (dict(page_tokens=1 << 17), zc.ERR_INVALID_ARG),
             (dict(n_seqs=0), zc.ERR_INVALID_ARG), (dict(n_heads=0), zc.ERR_INVALID_ARG), (dict(table_pages=0), zc.ERR_INVALID_ARG), (dict(n_pages=0), zc.ERR_INVALID_ARG),
             (dict(n_pages=1 << 31), zc.ERR_INVALID_ARG), (dict(table_pages=1 << 26), zc.ERR_INVALID_ARG), (dict(d_k_pages=None), zc.ERR_INVALID_ARG),
             (dict(d_v_pages=SOME + 8), zc.ERR_INVALID_ARG), (dict(d_table=None), zc.ERR_INVALID_ARG), (dict(d_lengths=None), zc.ERR_INVALID_ARG),
             (dict(d_table=SOME + 2), zc.ERR_INVALID_ARG), (dict(d_k_scales=SOME + 1), zc.ERR_INVALID_ARG)]


@pytest.mark.parametrize("change,status", BAD_CACHE)
def test_caches(change, status):
    assert attend(args(), cache(**change)) == status
    assert shared(args(), cache(n_seqs=1, d_lengths=2 * SOME), cache(**change)) == status
    change = {k: v for k, v in change.items()}
    assert evict(cache(**change), cache(d_lengths=2 * SOME)) == status
    assert evict(cache(d_lengths=2 * SOME), cache(**change)) == status
    assert zc.lib().zc_attend_workspace_bytes(C.byref(args()), None, C.byref(cache(**change))) == 0


@pytest.mark.parametrize("change", [dict(n_q_heads=0), dict(n_q_heads=7), dict(max_q_len=0), dict(n_tokens=4), dict(d_q=None), dict(d_out=None), dict(d_q=SOME + 8),
                                    dict(d_out=SOME + 2), dict(q_token_stride=1020), dict(out_head_stride=4), dict(scale=float("nan")), dict(scale=float("inf")),
                                    dict(reserved=1), dict(d_weights_out=SOME, d_lse=None), dict(d_weights_in=SOME), dict(max_prefix_len=5), dict(d_lse=SOME + 2),
                                    dict(n_tokens=1 << 29, d_q_start=SOME), dict(d_q_start=SOME + 1)])
def test_arguments_of_attention(change):
    assert attend(args(**change), cache()) == zc.ERR_INVALID_ARG


def test_other_refusals_of_attention():
    assert attend(None, cache()) == zc.ERR_INVALID_ARG and attend(args(), None) == zc.ERR_INVALID_ARG
    assert attend(args(struct_size=16), cache()) == zc.ERR_UNSUPPORTED
    pre = dict(n_seqs=1, d_lengths=2 * SOME)
    assert shared(args(), None, cache()) == zc.ERR_INVALID_ARG
    assert shared(args(), cache(), cache()) == zc.ERR_INVALID_ARG                               # a prefix of three sequences
    for other in (dict(format=zc.FMT_FP8_E5M2), dict(n_heads=1), dict(head_dim=64)):
        assert shared(args(), cache(**pre, **other), cache()) == zc.ERR_INVALID_ARG
    assert shared(args(d_weights_out=SOME), cache(**pre), cache()) == zc.ERR_INVALID_ARG
    assert shared(args(), cache(table_pages=(1 << 26) - 1, **pre), cache()) == zc.ERR_INVALID_ARG   # positions past 2^30


def test_workspace_is_asked_for():
    big = cache(table_pages=4096)
    need = zc.lib().zc_attend_workspace_bytes(C.byref(args()), None, C.byref(big))
    assert need > 0
    assert attend(args(), big, ws_bytes=need - 1) == zc.ERR_BUFFER_TOO_SMALL
    assert attend(args(), big, ws=None, ws_bytes=need) == zc.ERR_INVALID_ARG
    assert attend(args(), big, ws=SOME + 4, ws_bytes=need) == zc.ERR_INVALID_ARG


def test_eviction():
    to = dict(d_lengths=2 * SOME)
    assert evict(cache(), cache()) == zc.ERR_INVALID_ARG                                        # one array of lengths for both
    assert evict(cache(), cache(**to), sinks=15, recent=6) == zc.ERR_INVALID_ARG
    assert evict(cache(), cache(**to), sinks=0xFFFFFFFF, recent=0xFFFFFFFF) == zc.ERR_INVALID_ARG
    assert evict(cache(), cache(**to), w=None) == zc.ERR_INVALID_ARG
    assert evict(cache(), cache(**to), kept=None) == zc.ERR_INVALID_ARG
    assert evict(cache(), cache(**to), w_to=SOME) == zc.ERR_INVALID_ARG                         # weights onto themselves
    assert evict(cache(), cache(table_pages=1, **to), keep=17) == zc.ERR_BUFFER_TOO_SMALL
    for other in (dict(format=zc.FMT_FP8_E5M2), dict(n_heads=1), dict(head_dim=64), dict(n_seqs=2)):
        assert evict(cache(), cache(**to, **other)) == zc.ERR_INVALID_ARG


def paged(**change):
    x = dict(k_pages=torch.zeros((5, 16, 64), dtype=torch.uint8), v_pages=torch.zeros((5, 16, 64), dtype=torch.uint8), table=torch.zeros((2, 1, 2), dtype=torch.int32),
             lengths=torch.zeros(2, dtype=torch.int32), fmt=zc.FMT_FP8_E4M3)
    x.update(change)
    return zc.PagedCache(**x)


@pytest.mark.parametrize("change", [dict(table=torch.zeros((2, 1, 2), dtype=torch.int64)), dict(table=torch.zeros((2, 2), dtype=torch.int32)),
                                    dict(lengths=torch.zeros(3, dtype=torch.int32)), dict(v_pages=torch.zeros((4, 16, 64), dtype=torch.uint8)),
                                    dict(k_pages=torch.zeros((5, 16, 64), dtype=torch.int16)), dict(k_pages=torch.zeros((5, 16, 128), dtype=torch.uint8)[..., ::2]),
                                    dict(k_scales=torch.ones(2)), dict(v_scales=torch.ones((2, 1), dtype=torch.float64))])
def test_the_binding_checks_tensors(change):
    with pytest.raises(ValueError):
        paged(**change)


def test_the_binding_checks_the_calls_tensors():
    c = paged()
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    for bad in (q[:, :, :32], q.to(torch.float32), q[0]):
        with pytest.raises(ValueError):
            zc.attend(bad, c)
    with pytest.raises(ValueError):
        zc.attend(q, c, out=torch.zeros((2, 5, 64), dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        zc.attend(q, c, lse=torch.zeros((2, 4), dtype=torch.float64))
    with pytest.raises(ValueError):
        zc.attend(q, c, q_start=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        zc.attend(q, c, weights_out=torch.zeros((2, 1, 31)))
    with pytest.raises(ValueError):
        zc.evict(c, torch.zeros((2, 1, 31)), 4, paged())
    with pytest.raises(ValueError):
        zc.evict(c, torch.zeros((2, 1, 32)), 4, paged(), kept=torch.zeros((2, 1, 5), dtype=torch.int32))
    with pytest.raises(ValueError):
        zc.attend(q.to(torch.float16), c)
    with pytest.raises(ValueError):
        zc.attend(q, c)                                          # not on a GPU
    with pytest.raises(ValueError):
        zc.evict(c, torch.zeros((2, 1, 32)), 4, paged())
    for other in (torch.float8_e5m2, torch.float8_e4m3fnuz):
        with pytest.raises(ValueError):
            paged(k_pages=torch.zeros((5, 16, 64), dtype=other))
    with pytest.raises(zc.ZcError):
        paged(fmt=zc.FMT_FP4_E2M1_MX)


def test_calls_too_large_for_a_launch():
    wide = dict(n_seqs=1 << 20, n_heads=2)
    assert attend(args(n_tokens=1 << 20, n_q_heads=64, max_q_len=1), cache(n_seqs=1 << 20, n_heads=64)) == zc.ERR_INVALID_ARG
    assert evict(cache(table_pages=1 << 20, **wide), cache(d_lengths=2 * SOME, table_pages=1 << 20, **wide), keep=1 << 24) == zc.ERR_INVALID_ARG
