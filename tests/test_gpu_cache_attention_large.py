"""Attention over the cache, and in tiles over packed sequences, where numbers are
large: queries at the end of bfloat16's range over keys of zero (4 bits), and scores
up to 2^26, where half a unit in a score's last place is a factor that the weights
have to have room for.  Such weights are not exact, but every output is one of its
values' means: it lies between the smallest and the largest of them, give or take its
rounding."""
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


SIZES = pytest.mark.parametrize("size", [s * 2.0 ** e for e in (10, 18, 21, 22, 23, 26) for s in (1, -1)])


def between(o, v):
    """o: [rows, dim] from values [keys, dim]: two roundings to the type, 2^-8 each, of the largest."""
    lo, hi = v.amin(0), v.amax(0)
    t = 2.0 ** -7 * torch.maximum(lo.abs(), hi.abs())
    return bool(torch.isfinite(o).all()) and bool(((o.double() >= lo - t) & (o.double() <= hi + t)).all())


@SIZES
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
def test_large_scores(sg, dtype, bits, size):
    lens, dim = [900, 300, 17], 128
    for heads in (8, 16):
        cache, table = made(sg, 42, lens, 16, 2, dim, dtype, bits)
        q = (queries(42, 3, heads, dim, dtype).float() * 0.01 + (1 if size > 0 else -1)).to(dtype)
        if bits == 16:
            cache.k.mul_(2.0 ** -6).add_(1.0)
        else:
            cache.k.fill_(0xFF)                            # codes of 7
            cache.k_scale.fill_(1 / 7)
        o, lse = sg.sync_cache_attn(cache, q, table, i32(lens), scale=abs(size) / dim, lse=True)
        assert bool(torch.isfinite(lse).all())
        for s, n in enumerate(lens):
            v, _ = ref.values(cache, "v", table[s], n)
            assert all(between(o[s, h:h + 1], v[:, h // (heads // 2)]) for h in range(heads))


@SIZES
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "cross"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
def test_large_scores_in_tiles(sg, dtype, causal, size):
    g = torch.Generator(device="cuda").manual_seed(43)
    q = (torch.randn((300, 4, 128), generator=g, device="cuda") * 0.01 + (1 if size > 0 else -1)).to(dtype)
    k = (torch.randn((1500, 2, 128), generator=g, device="cuda") * 2.0 ** -6 + 1).to(dtype)
    v = torch.randn((1500, 2, 128), generator=g, device="cuda").to(dtype)
    plan = sg.sync_attn_plan([300], [1500], 4, 2, 128, dtype, train=True, causal=causal)
    o, lse = sg.sync_attn_forward(plan, q, k, v, scale=abs(size) / 128, lse=True)
    assert bool(torch.isfinite(lse).all()) and all(between(o[:, h], v[:, h // 2].double()) for h in range(4))
    plan.check()
    plan.close()
