"""How the attention calls take their arguments, against the definition in 64 bits (tests/paged.py)."""
import pytest
import torch

from paper_2508_19263_amd import zc
from tests.paged import Cache, agree, attention, starts
from tests.test_gpu_attend import queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q_lens", [[1, 1, 1], [5, 1, 40], [0, 300, 2]])
@pytest.mark.parametrize("shared", [False, True])
def test_all_query_tokens_are_answered_whatever_their_number(q_lens, shared):
    """Where it is not said how many query tokens a sequence has at most, it may have any number of those there are."""
    cache = Cache([70, 9, 400], 2, 128, zc.FMT_FP8_E4M3)
    prefix = Cache([100], 2, 128, zc.FMT_FP8_E4M3, seed=3) if shared else None
    q = queries(sum(q_lens), 8, 128)
    out, lse = torch.full_like(q, 3.0), torch.full((sum(q_lens), 8), 3.0, device="cuda")
    if shared:
        zc.attend_shared(q, prefix.paged, cache.paged, q_start=starts(q_lens), out=out, lse=lse)
    else:
        zc.attend(q, cache.paged, q_start=starts(q_lens), out=out, lse=lse)
    want, want_lse, _, tol, tol_lse, _ = attention(q, q_lens, cache, prefix)
    agree(out, want, tol, "out")
    agree(lse, want_lse, tol_lse, "lse")


@pytest.mark.parametrize("n,heads", [(1, 8), (3, 1), (1, 1)])
def test_strides_of_single_tokens_and_heads(n, heads):
    """Where there is only one token, or one query head, its stride is any number, and no element is found by it."""
    cache = Cache([200] * n, min(heads, 2), 64, zc.FMT_BF16)
    flat = queries(n, heads, 64)
    want, want_lse = zc.attend(flat, cache.paged)
    order = (2, 0, 1) if n == 1 else (0, 2, 1)                   # a last dimension of one element goes where there is only one token or head
    q, out = (torch.zeros((heads, 64, 1) if n == 1 else (n, 64, 1), dtype=torch.bfloat16, device="cuda").permute(order) for _ in range(2))
    q.copy_(flat)
    assert q.shape == flat.shape and (q.stride(0) % 8 or q.stride(1) % 8) and q.stride(2) == 1
    got, lse = zc.attend(q, cache.paged, out=out)
    assert torch.equal(got, want) and torch.equal(lse, want_lse) and got is out
