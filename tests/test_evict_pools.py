"""zc_evict to a cache whose keys and values have one pool, from one where they lie apart, is refused before anything is queued (no GPU needed)."""
import pytest

from paper_2508_19263_amd import zc
from tests.test_kv_rows_arguments import FP4, SOME, cache, cache4, evict

APART = dict(d_k_pages=SOME, d_v_pages=2 * SOME)
FEW = dict(table_pages=1)                                      # room for less than what stays: the last thing that is refused


@pytest.mark.parametrize("fmt", [zc.FMT_BF16, zc.FMT_FP8_E4M3])
def test_one_pool_for_keys_and_values(fmt):
    kind = dict(format=fmt)
    for source, change, status in ((APART, APART, zc.ERR_BUFFER_TOO_SMALL), (APART, {}, zc.ERR_INVALID_ARG), ({}, {}, zc.ERR_BUFFER_TOO_SMALL), ({}, APART, zc.ERR_BUFFER_TOO_SMALL)):
        assert evict(cache(**dict(kind, **source)), cache(d_lengths=2 * SOME, **dict(kind, **change, **FEW))) == status, (source, change)


@pytest.mark.parametrize("fmt", FP4)
def test_one_pool_of_block_scales(fmt):
    own = dict(APART, d_k_block_scales=SOME, d_v_block_scales=2 * SOME)
    for change, status in ((dict(), zc.ERR_BUFFER_TOO_SMALL), (dict(d_v_block_scales=SOME), zc.ERR_INVALID_ARG), (dict(d_v_pages=SOME), zc.ERR_INVALID_ARG)):
        assert evict(cache4(fmt, **own), cache4(fmt, **dict(own, d_lengths=2 * SOME, **change, **FEW))) == status, change
