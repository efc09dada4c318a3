"""The binding imports with a torch that lacks the newest element types: the codec needs none of them, and pages can be held as plain integers."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import torch
for name in %r:
    if hasattr(torch, name):
        delattr(torch, name)
from paper_2508_19263_amd import zc
zc.lib()
for fmt in (zc.FMT_FP4_E2M1_MX, zc.FMT_FP4_E2M1_NV):
    pages, blocks = torch.zeros((3, 16, 32), dtype=torch.uint8), torch.zeros((3, 16, 64 // zc.scale_block(fmt)), dtype=torch.uint8)
    table, lengths = torch.zeros((1, 1, 3), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    assert zc.PagedCache(pages, pages.clone(), table, lengths, fmt, k_blocks=blocks, v_blocks=blocks.clone()).head_dim == 64
print("imported")
"""


@pytest.mark.parametrize("missing", [("float4_e2m1fn_x2",), ("float8_e8m0fnu",), ("float4_e2m1fn_x2", "float8_e8m0fnu")])
def test_types_that_a_torch_may_lack(missing):
    r = subprocess.run([sys.executable, "-c", PROGRAM % (missing,)], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0 and "imported" in r.stdout, r.stderr[-2000:]
