"""The built library's attention kernels over K/V pages: which there are, and how they load pages."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2508_19263_amd import zc

LLVM = "/opt/rocm/llvm/bin"
ROW_BYTES = {zc.FMT_BF16: 2.0, zc.FMT_FP8_E4M3: 1.0, zc.FMT_FP8_E5M2: 1.0, zc.FMT_FP4_E2M1_MX: 0.5, zc.FMT_FP4_E2M1_NV: 0.5}     # per element


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{(format, head_dim, tiles, logits, last template argument): listing} of k_attend_few."""
    if not os.path.exists(LLVM + "/llvm-objdump"):
        pytest.skip("llvm-objdump not found")
    zc.lib()                                                   # (fails if the library is not built)
    folder = str(tmp_path_factory.mktemp("kernels"))
    shutil.copy(os.path.join(os.path.dirname(zc.__file__), "libzc.so"), folder)
    subprocess.run([LLVM + "/llvm-objdump", "--offloading", "libzc.so"], cwd=folder, check=True, capture_output=True)
    found = {}
    for f in sorted(f for f in os.listdir(folder) if f.endswith("gfx950")):
        names = set(subprocess.run([LLVM + "/llvm-readelf", "-s", "--wide", f], cwd=folder, check=True, capture_output=True, text=True).stdout.split())
        for name in names:
            m = re.match(r"_ZN2zc\d+_GLOBAL__N_1\d+k_attend_fewILi(\d+)ELi(\d+)ELi(\d)ELb([01])EL.*?(\d)EEE", name)
            if m and "." not in name:
                found[tuple(int(x) for x in m.groups())] = subprocess.run([LLVM + "/llvm-objdump", "-d", "--no-show-raw-insn", "--disassemble-symbols=" + name, f],
                                                                          cwd=folder, check=True, capture_output=True, text=True).stdout
    assert len(found) >= 40
    return found


def test_no_build_loads_short_rows_past_the_caches(kernels):
    """Rows of less than 64 bytes never go there, so no kernel is built for it."""
    for (fmt, dim, _, _, _), listing in kernels.items():
        assert ROW_BYTES[fmt] * dim >= 64 or not re.search(r"buffer_load.* nt\b", listing), (fmt, dim)
    assert any(re.search(r"buffer_load.* nt\b", listing) for listing in kernels.values())


@pytest.mark.parametrize("fmt", [zc.FMT_BF16, zc.FMT_FP8_E4M3, zc.FMT_FP8_E5M2])
def test_kernels_that_load_past_the_caches_can_load_through_them(kernels, fmt):
    """BF16 and FP8: what a call reads is known when the lengths and the table are, on the device, so no kernel can only go past the caches."""
    both = 0
    for key, listing in kernels.items():
        loads = re.findall(r"buffer_load_(?:dword|dwordx2|dwordx4) .*", listing)
        past = [x for x in loads if re.search(r" nt\b", x)]
        if key[0] == fmt and past:
            assert len(loads) >= 2 * len(past), (key, len(loads), len(past))
            both += 1
    assert both == 8                                           # two sizes of heads, one tile or two, with logits or without
