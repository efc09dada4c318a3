"""The example that takes a K/V cache through the codec, attention and eviction."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "kv_cache.py")


def test_example():
    spec = importlib.util.spec_from_file_location("kv_cache_example", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(prompt=512, answers=3, steps=20, keep=128, quiet=True)
    assert r["lengths"].tolist() == [128] and bool(r["out"].isfinite().all()) and bool(r["near"].isfinite().all())
    kept = r["kept"][0]
    assert bool((kept[:, 1:] > kept[:, :-1]).all()) and bool((kept[:, :4] == torch.arange(4, device="cuda")).all())
    assert bool((kept[:, -32:] == torch.arange(480, 512, device="cuda")).all())
    # a quarter of the tokens, the heaviest of most, has more than its share of the weight
    assert r["share"] > 0.3
