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
