"""zc_kv_write into a cache whose keys and values have one pool is refused before anything is queued (no GPU needed: no address is followed)."""
import pytest

from paper_2508_19263_amd import zc
from tests.test_kv_rows_arguments import FP4, SOME, cache, cache4, call, rows

# n_tokens = 0 shows what is refused without a launch
NONE = dict(n_tokens=0, d_q_start=SOME)


@pytest.mark.parametrize("fmt", [zc.FMT_BF16, zc.FMT_FP8_E4M3, zc.FMT_FP8_E5M2])
def test_one_pool_for_keys_and_values(fmt):
    apart = cache(format=fmt, d_v_pages=2 * SOME, d_k_pages=SOME)
    one = cache(format=fmt, d_v_pages=SOME, d_k_pages=SOME)
    assert call("zc_kv_write", rows(**NONE), apart) == zc.OK
    assert call("zc_kv_write", rows(**NONE), one) == zc.ERR_INVALID_ARG
    assert call("zc_kv_read", rows(**NONE), one) == zc.OK        # (reading does no harm)


@pytest.mark.parametrize("fmt", FP4)
def test_one_pool_of_block_scales(fmt):
    for change, status in ((dict(), zc.OK), (dict(d_v_block_scales=SOME), zc.ERR_INVALID_ARG), (dict(d_v_pages=SOME), zc.ERR_INVALID_ARG)):
        c = cache4(fmt, **dict(dict(d_k_pages=SOME, d_v_pages=2 * SOME, d_k_block_scales=SOME, d_v_block_scales=2 * SOME), **change))
        assert call("zc_kv_write", rows(**NONE), c) == status, change


@pytest.mark.parametrize("change,status", [(dict(), zc.OK), (dict(d_v=2 * SOME), zc.ERR_INVALID_ARG), (dict(v_token_stride=512), zc.ERR_INVALID_ARG), (dict(v_head_stride=64), zc.ERR_INVALID_ARG)])
def test_keys_that_are_the_values(change, status):
    """The same rows under the same scales are the same bits in one pool."""
    c = cache(d_k_pages=SOME, d_v_pages=SOME)
    assert call("zc_kv_write", rows(**dict(dict(NONE, d_k=SOME, d_v=SOME), **change)), c) == status
    for scales, same in (((SOME, SOME), zc.OK), ((SOME, 2 * SOME), zc.ERR_INVALID_ARG), ((SOME, None), zc.ERR_INVALID_ARG)):
        c = cache(format=zc.FMT_FP8_E4M3, d_k_pages=SOME, d_v_pages=SOME, d_k_scales=scales[0], d_v_scales=scales[1])
        assert call("zc_kv_write", rows(**dict(NONE, d_k=SOME, d_v=SOME)), c) == same
