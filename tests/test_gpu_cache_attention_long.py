"""Attention over the cache in 4 bits where a warp adds up hundreds of thousands of
tokens of equal weight: nothing larger than the result may be carried along (the
codes are stored with 8 added).

Each product of 16 tokens is added in 32 bits, cut at 2^-23 of what is there: the sum
so far, at most the largest sum of any run of tokens, M code units, and up to 16
codes of 15.  For n tokens of weight 1 / n, n / 8 additions (codes, and the 8 off
them) leave at most n / 8 * 2^-23 * (M + 240) / n scales in an entry; weights of
2^11 and their products with one scale are exact otherwise, and the result is rounded
once."""
import pytest
import torch

from tests import cache_reference as ref
from tests.test_gpu_cache import i32
from tests.test_gpu_cache_attention_range import packed_codes

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("n,heads,kv,dim", [(16384, 32, 8, 128), (65536, 12, 1, 64), (262144, 32, 8, 128), (262144, 32, 8, 96)])
def test_flat_rows(sg, n, heads, kv, dim, dtype):
    page, seqs, scale = 64, 300, torch.tensor(0.2).half().item()       # (no power of two, whose multiples add exactly)
    cache = sg.sync_kv_cache(n // page, page, kv, dim, dtype, bits=4)
    g = torch.Generator(device="cuda").manual_seed(61)
    for t in (cache.k, cache.v):
        t.copy_(packed_codes(torch.randint(-7, 8, t.shape[:3] + (dim,), generator=g, device="cuda", dtype=torch.int8)))
    cache.k_scale.fill_(scale)
    cache.v_scale.fill_(scale)
    table = torch.arange(n // page, device="cuda", dtype=torch.int32).expand(seqs, -1).contiguous()   # all read the same
    q = torch.zeros((seqs, heads, dim), device="cuda", dtype=dtype)
    o = sg.sync_cache_attn(cache, q, table, i32([n] * seqs))
    u, pages = torch.finfo(dtype).eps / 2, table[0].long()
    for h in range(kv):
        codes = (ref.decoded(cache.v[pages, h], cache.v_scale[pages, h]) / scale).view(n, dim)
        want, sums = scale * codes.mean(0), codes.cumsum(0)
        m = (sums.amax(0).clamp(min=0) - sums.amin(0).clamp(max=0)).amax().item()
        cut = 2.0 ** -26 * (m + 240) * scale
        for s in (0, 137, seqs - 1):
            off = (o[s, h * (heads // kv):(h + 1) * (heads // kv)].double() - want).abs()
            worst = (off / (cut + u * want.abs())).amax().item()
            assert worst <= 1, f"head {h}: {worst} times what is allowed; the mean is off by {(off.mean() / want.abs().mean()).item()}"
