"""What the calls over K/V pages refuse beside tests/test_paged_arguments.py, and how much scratch they ask for (no GPU needed: nothing is
queued, no address is followed).  The binding's refusals are told apart by their messages: without a GPU every call is refused in the end."""
import ctypes as C

import pytest
import torch

from paper_2508_19263_amd import zc
from tests.test_paged_arguments import SOME, args, cache, paged


def call(**change):
    x = dict(q=torch.zeros((2, 4, 64), dtype=torch.bfloat16), cache=paged())
    x.update(change)
    return zc.attend(**x)


def evict(**change):
    x = dict(cache=paged(), weights=torch.zeros((2, 1, 32)), keep=4, into=paged())
    x.update(change)
    return zc.evict(**x)


@pytest.mark.parametrize("ws", [torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(1 << 20, dtype=torch.uint8)[::2]])
def test_scratch_with_holes(ws):
    """Its size is taken from the number of elements, so these have to lie one behind the other."""
    with pytest.raises(ValueError, match="ws"):
        call(ws=ws)


@pytest.mark.parametrize("name", ["max_q_len", "window", "sinks", "max_kv_len"])
@pytest.mark.parametrize("value", [-1, 1 << 32, (1 << 32) + 5])
def test_numbers_that_the_call_has_no_room_for(name, value):
    """ctypes would cut them to 32 bits: sinks=-1 would make every token a sink."""
    with pytest.raises(ValueError, match=name):
        call(**{name: value})
    with pytest.raises(ValueError, match=name):
        zc.attend_shared(torch.zeros((2, 4, 64), dtype=torch.bfloat16), paged(table=torch.zeros((1, 1, 2), dtype=torch.int32), lengths=torch.zeros(1, dtype=torch.int32)),
                         paged(), **{name: value})


@pytest.mark.parametrize("name", ["keep", "sinks", "recent"])
@pytest.mark.parametrize("value", [-1, 1 << 32])
def test_numbers_that_eviction_has_no_room_for(name, value):
    with pytest.raises(ValueError, match=name):
        evict(**{name: value})


def test_gradients_are_not_dropped():
    q, w = torch.zeros((2, 4, 64), dtype=torch.bfloat16, requires_grad=True), torch.zeros((2, 1, 32), requires_grad=True)
    with pytest.raises(ValueError, match="gradient"):
        call(q=q)
    with pytest.raises(ValueError, match="gradient"):
        call(weights=w, weights_out=torch.zeros((2, 1, 32)))
    with pytest.raises(ValueError, match="gradient"):
        evict(weights=w, into_weights=torch.zeros((2, 1, 32)))
    with torch.no_grad():
        with pytest.raises(ValueError, match="GPU"):             # nothing but that is wrong
            call(q=q)
        with pytest.raises(ValueError, match="GPU"):
            evict(weights=w)


@pytest.mark.parametrize("out", [torch.zeros((1, 4, 64), dtype=torch.bfloat16).expand(2, 4, 64), torch.zeros((2, 1, 64), dtype=torch.bfloat16).expand(2, 4, 64),
                                 torch.zeros(1000, dtype=torch.bfloat16).as_strided((2, 4, 64), (256, 32, 1))])
def test_results_on_top_of_each_other(out):
    with pytest.raises(ValueError, match="overlap"):
        call(out=out)


def test_queries_that_are_read_again():
    """Weights of many rows come from the queries once more, when the results have been written."""
    for rows in (1, 100):
        x = args(n_tokens=100, max_q_len=rows, d_q_start=SOME, d_weights_out=4 * SOME, d_out=2 * SOME)
        c = cache(table_pages=4096)
        need = zc.lib().zc_attend_workspace_bytes(C.byref(x), None, C.byref(c))
        assert zc.lib().zc_attend(C.byref(x), C.byref(c), 8 * SOME, max(need, 1) - 1, None) == zc.ERR_BUFFER_TOO_SMALL       # nothing but that is wrong
        x.d_out = x.d_q
        assert zc.lib().zc_attend(C.byref(x), C.byref(c), 8 * SOME, 1 << 40, None) == zc.ERR_INVALID_ARG


def scratch(x, c):
    return zc.lib().zc_attend_workspace_bytes(C.byref(x), None, C.byref(c))


def weighed(**change):
    return args(d_q_start=SOME, d_out=2 * SOME, d_weights_out=4 * SOME, **change)


def test_scratch_follows_the_longest_length_and_not_the_tables_room():
    """One prompt of 300 tokens: sums of parts of the rows, for 300 tokens each."""
    x = weighed(n_tokens=300, n_q_heads=32, max_q_len=300, max_kv_len=300)
    small, large = (scratch(x, cache(n_seqs=1, n_heads=8, table_pages=n)) for n in (19, 1 << 16))
    assert 0 < small == large < 1 << 20


def test_scratch_of_weights_has_a_bound():
    """Logits of few rows are kept for the weights where they take at most 1 GiB; else the keys are read again, with 32 bits for every token and
    as many parts of the rows as make about 1,024 workgroups."""
    large = cache(n_seqs=32, n_heads=8, table_pages=8192)                      # room for 131,072 tokens
    parts = 32 * 8 * 24 * 16 * (128 * 4 + 8)                                   # of the attention: rows x parts of 8,192 tokens
    x = weighed(n_tokens=96, n_q_heads=64, max_q_len=3)                        # 24 rows: 3 GiB of logits
    assert scratch(x, large) <= parts + 1024
    x.max_kv_len = 8000                                                        # 188 MiB
    assert scratch(x, large) >= 32 * 8 * 24 * 8000 * 4
    x = weighed(n_tokens=32, n_q_heads=8, max_q_len=1)                         # one row: 128 MiB
    assert scratch(x, large) >= 32 * 8 * 131072 * 4
    x = weighed(n_tokens=1, n_q_heads=24, max_q_len=1)                         # one cache, 24 rows, just 1 GiB and a step more
    for tokens, fits in ((11184800, True), (11184832, False)):
        c = cache(n_seqs=1, n_heads=1, table_pages=tokens // 16)
        need, logits = scratch(x, c), 24 * tokens * 4
        assert (need >= logits) == fits and need < logits + (1 << 25) and (fits or need < 1 << 30)
