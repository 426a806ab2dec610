"""Attention over the cache in 4 bits for queries at the end of bfloat16's range:
scores stay small where the keys are zero."""
import pytest
import torch

from tests import cache_reference as ref
from tests.test_gpu_cache import i32
from tests.test_gpu_cache_attention import made, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


@pytest.mark.parametrize("heads", [8, 24])
@pytest.mark.parametrize("gain", [1.0, 2.0 ** 100, 2.0 ** 124])
def test_zero_keys(sg, gain, heads):
    lens = [300, 33]
    cache, table = made(sg, 41, lens, 16, 2, 64, torch.bfloat16, 4)
    cache.k_scale.zero_()
    q = (queries(41, 2, heads, 64, torch.bfloat16).float() * gain).bfloat16()
    assert bool(torch.isfinite(q).all())
    ref.check(sg.sync_cache_attn(cache, q, table, i32(lens), lse=True), ref.attention(cache, q, table, lens, None, 0.125))
