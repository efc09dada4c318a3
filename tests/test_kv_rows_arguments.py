"""What zc_kv_write and zc_kv_read refuse, and what 4-bit caches have to have, before anything is queued (no GPU needed: no address is followed)."""
import ctypes as C

import pytest
import torch

from paper_2508_19263_amd import zc
from tests.test_paged_arguments import BAD_CACHE, SOME, args, attend, cache, evict, shared

FP4 = [zc.FMT_FP4_E2M1_MX, zc.FMT_FP4_E2M1_NV]
CALLS = ["zc_kv_write", "zc_kv_read"]


def rows(**change):
    r = zc.KvRows()
    r.struct_size = C.sizeof(zc.KvRows)
    r.n_tokens, r.d_k, r.d_v = 3, SOME, 2 * SOME
    r.k_token_stride = r.v_token_stride = 256
    r.k_head_stride = r.v_head_stride = 128
    for name, v in change.items():
        setattr(r, name, v)
    return r


def call(name, r, c):
    return getattr(zc.lib(), name)(C.byref(r) if r is not None else None, C.byref(c) if c is not None else None, None)


def cache4(fmt, **change):
    return cache(**dict(dict(format=fmt, d_k_block_scales=SOME, d_v_block_scales=SOME), **change))


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("change,status", BAD_CACHE)
def test_caches(name, change, status):
    assert call(name, rows(), cache(**change)) == status


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("change", [dict(n_tokens=4), dict(n_tokens=2), dict(d_k=None), dict(d_v=None), dict(d_k=SOME + 8), dict(d_v=SOME + 2), dict(k_token_stride=252),
                                    dict(v_head_stride=4), dict(d_q_start=SOME + 2), dict(n_tokens=1 << 30, d_q_start=SOME)])
def test_rows(name, change):
    assert call(name, rows(**change), cache()) == zc.ERR_INVALID_ARG


@pytest.mark.parametrize("name", CALLS)
def test_other_refusals(name):
    assert call(name, None, cache()) == zc.ERR_INVALID_ARG and call(name, rows(), None) == zc.ERR_INVALID_ARG
    assert call(name, rows(struct_size=8), cache()) == zc.ERR_UNSUPPORTED
    assert call("zc_kv_read", rows(d_v=SOME), cache()) == zc.ERR_INVALID_ARG     # keys and values to one place
    assert call(name, rows(n_tokens=0, d_q_start=SOME, d_k=None, d_v=None), cache()) == zc.OK


@pytest.mark.parametrize("fmt", FP4)
@pytest.mark.parametrize("change,status", [(dict(d_k_block_scales=None), zc.ERR_UNSUPPORTED), (dict(d_v_block_scales=None), zc.ERR_UNSUPPORTED),
                                           (dict(d_k_block_scales=SOME + 8), zc.ERR_INVALID_ARG), (dict(d_v_block_scales=SOME + 4), zc.ERR_INVALID_ARG),
                                           (dict(struct_size=zc.KvCache.d_k_block_scales.offset), zc.ERR_UNSUPPORTED), (dict(head_dim=96), zc.ERR_UNSUPPORTED)])
def test_caches_of_four_bits(fmt, change, status):
    c = cache4(fmt, **change)
    for name in CALLS:
        assert call(name, rows(), c) == status
    assert attend(args(), c) == status
    assert shared(args(), cache4(fmt, n_seqs=1, d_lengths=2 * SOME), c) == status
    assert evict(c, cache4(fmt, d_lengths=2 * SOME)) == status and evict(cache4(fmt, d_lengths=2 * SOME), c) == status
    assert zc.lib().zc_attend_workspace_bytes(C.byref(args()), None, C.byref(c)) == 0


def test_block_scales_of_formats_that_have_none():
    for change in (dict(d_k_block_scales=SOME), dict(d_v_block_scales=SOME)):
        assert attend(args(), cache(**change)) == zc.ERR_UNSUPPORTED
        assert call("zc_kv_write", rows(), cache(**change)) == zc.ERR_UNSUPPORTED


def test_callers_that_know_the_first_layout_of_a_cache():
    """zc_kv_cache has grown at its end: without its last two members it is taken as before."""
    big, old = cache(table_pages=4096), cache(table_pages=4096, struct_size=zc.KvCache.d_k_block_scales.offset, d_k_block_scales=SOME, d_v_block_scales=SOME)
    need = zc.lib().zc_attend_workspace_bytes(C.byref(args()), None, C.byref(big))
    assert need > 0 and zc.lib().zc_attend_workspace_bytes(C.byref(args()), None, C.byref(old)) == need
    assert attend(args(), old, ws_bytes=need - 1) == zc.ERR_BUFFER_TOO_SMALL       # nothing but that is wrong


def test_formats_are_not_mixed():
    a, b = (cache4(fmt, d_lengths=n * SOME) for n, fmt in zip((1, 2), FP4))
    assert evict(a, b) == zc.ERR_INVALID_ARG and evict(cache(), b) == zc.ERR_INVALID_ARG
    assert shared(args(), cache4(FP4[0], n_seqs=1, d_lengths=2 * SOME), cache4(FP4[1])) == zc.ERR_INVALID_ARG


def paged(fmt=zc.FMT_FP8_E4M3, **change):
    packed, block = (2, zc.scale_block(fmt)) if fmt in FP4 else (1, 0)
    x = dict(k_pages=torch.zeros((5, 16, 64 // packed), dtype=torch.uint8), v_pages=torch.zeros((5, 16, 64 // packed), dtype=torch.uint8),
             table=torch.zeros((2, 1, 2), dtype=torch.int32), lengths=torch.zeros(2, dtype=torch.int32), fmt=fmt)
    if block:
        x.update(k_blocks=torch.zeros((5, 16, 64 // block), dtype=torch.uint8), v_blocks=torch.zeros((5, 16, 64 // block), dtype=torch.uint8))
    x.update(change)
    return zc.PagedCache(**x)


@pytest.mark.parametrize("fmt", FP4)
def test_the_binding_checks_block_scales(fmt):
    c = paged(fmt)
    assert c.head_dim == 64 and c.c.head_dim == 64 and c.c.d_k_block_scales == c.k_blocks.data_ptr()
    n = 64 // zc.scale_block(fmt)
    for bad in (None, torch.zeros((5, 16, n + 1), dtype=torch.uint8), torch.zeros((5, 16, n)), torch.zeros((4, 16, n), dtype=torch.uint8), torch.zeros((5, 16, 2 * n), dtype=torch.uint8)[..., ::2]):
        for name in ("k_blocks", "v_blocks"):
            with pytest.raises(ValueError):
                paged(fmt, **{name: bad})
    with pytest.raises(zc.ZcError):
        paged(fmt, k_blocks=None, v_blocks=None)
    with pytest.raises(ValueError):
        paged(k_blocks=torch.zeros((5, 16, n), dtype=torch.uint8))
    own = {zc.FMT_FP4_E2M1_MX: torch.float8_e8m0fnu, zc.FMT_FP4_E2M1_NV: torch.float8_e4m3fn}[fmt]
    paged(fmt, k_blocks=c.k_blocks.view(own), k_pages=c.k_pages.view(torch.float4_e2m1fn_x2))
    with pytest.raises(ValueError):
        paged(fmt, k_blocks=c.k_blocks.view(torch.float8_e5m2))


def some(**change):
    return torch.zeros(change.pop("shape", (2, 1, 64)), dtype=change.pop("dtype", torch.bfloat16), **change)


def test_the_binding_checks_rows():
    c = paged()
    for bad in (some(shape=(2, 1, 32)), some(dtype=torch.float32), some(dtype=torch.float16), some(shape=(2, 64)), some(shape=(2, 2, 64)), some(shape=(3, 1, 64)),
                some(shape=(2, 1, 128))[..., ::2]):
        with pytest.raises(ValueError):
            zc.write_kv(bad, some(), c)
        with pytest.raises(ValueError):
            zc.write_kv(some(), bad, c)
        with pytest.raises(ValueError):
            zc.read_kv(c, v=bad, k=some())
    for start in (torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64), torch.zeros(6, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError, match="q_start"):
            zc.write_kv(some(), some(), c, start)
    with pytest.raises(ValueError, match="n_tokens"):
        zc.read_kv(c, torch.zeros(3, dtype=torch.int32))
    for n in (-1, 1 << 32):
        with pytest.raises(ValueError, match="n_tokens"):
            zc.read_kv(c, torch.zeros(3, dtype=torch.int32), n)
    with pytest.raises(ValueError, match="q_start"):
        zc.read_kv(c, n_tokens=3)
    with pytest.raises(ValueError, match="GPU"):
        zc.write_kv(some(), some(), c)
    with pytest.raises(ValueError, match="GPU"):
        zc.read_kv(c)


def test_gradients_are_not_dropped():
    c, wants = paged(), some(requires_grad=True)
    for k, v in ((wants, some()), (some(), wants)):
        with pytest.raises(ValueError, match="gradient"):
            zc.write_kv(k, v, c)
    with torch.no_grad():
        with pytest.raises(ValueError, match="GPU"):             # nothing but that is wrong
            zc.write_kv(wants, wants, c)


@pytest.mark.parametrize("out", [some(shape=(1, 1, 64)).expand(2, 1, 64), some(shape=(1000,)).as_strided((2, 1, 64), (32, 64, 1))])
def test_results_on_top_of_each_other(out):
    with pytest.raises(ValueError, match="overlap"):
        zc.read_kv(paged(), k=out)


def test_heads_on_top_of_the_next_token():
    c = paged(table=torch.zeros((2, 2, 2), dtype=torch.int32))
    with pytest.raises(ValueError, match="overlap"):             # token 1's first head is token 0's second
        zc.read_kv(c, k=some(shape=(1000,)).as_strided((2, 2, 64), (64, 64, 1)))
    for shape, strides in (((2, 2, 64), (128, 64, 1)), ((2, 2, 64), (64, 128, 1))):
        with pytest.raises(ValueError, match="GPU"):
            zc.read_kv(c, k=some(shape=(1000,)).as_strided(shape, strides))


def meet(k, v):
    """The elements that two tensors have in common, one by one."""
    a, b = (set((t.data_ptr() // 2 + torch.cat([torch.arange(t.shape[2]) + i * t.stride(0) + j * t.stride(1) for i in range(t.shape[0]) for j in range(t.shape[1])])).tolist())
            for t in (k, v))
    return bool(a & b)


@pytest.mark.parametrize("shape", [(1, 1), (1, 3), (2, 1), (2, 2), (5, 3)])
@pytest.mark.parametrize("k_strides", [(200, 64), (64, 400), (720, 72), (400, 128), (136, 680)])
def test_keys_on_top_of_values(shape, k_strides):
    """Every place of V's first row around K's, with K's strides and with others: what has elements in common is refused, what goes between is not."""
    room, (n, heads) = some(shape=(40000,)), shape
    c = paged(table=torch.zeros((2, heads, 2), dtype=torch.int32))
    start, seen = torch.zeros(3, dtype=torch.int32), set()
    if (n > 1 and heads > 1) and not (k_strides[0] >= k_strides[1] * (heads - 1) + 64 or k_strides[1] >= k_strides[0] * (n - 1) + 64):
        return                                                   # (K's own rows would overlap)
    for v_strides in (k_strides, (k_strides[0] * 2 + 8, k_strides[1] * 2 + 8)):
        if n > 1 and heads > 1 and not (v_strides[0] >= v_strides[1] * (heads - 1) + 64 or v_strides[1] >= v_strides[0] * (n - 1) + 64):
            continue
        k = room.as_strided((n, heads, 64), k_strides + (1,), 20000)
        for off in list(range(-1600, 1601, 8)) + [-65, -63, 63, 65]:
            v = room.as_strided((n, heads, 64), v_strides + (1,), 20000 + off)
            both = meet(k, v)
            seen.add(both)
            with pytest.raises(ValueError, match="rows of k and v overlap" if both else "GPU"):
                zc.read_kv(c, start, k=k, v=v)
    assert seen == {True, False}


def test_packed_arguments_are_the_structures():
    """The binding packs a call's arguments itself: every member is where the structure has it."""
    for kind, pack in ((zc.KvRows, zc._pack_kv_rows), (zc.AttendArgs, zc._pack_attend_args)):
        values = [i + 1 for i in range(len(kind._fields_))]
        a = kind.from_buffer_copy(pack(*values))
        assert [getattr(a, name) for name, _ in kind._fields_] == values and len(pack(*values)) == C.sizeof(kind)
