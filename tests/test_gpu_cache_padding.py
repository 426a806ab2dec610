"""Rows of a step that belong to no sequence, in front of the first one as behind
the last: kept in tensors that are given, zero where the call is asked to fill them."""
import math

import pytest
import torch

from tests import cache_reference as ref
from tests.test_gpu_cache import i32
from tests.test_gpu_cache_attention import BITS, made, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


@BITS
@pytest.mark.parametrize("starts", [[3, 4, 4, 6], [300, 301, 301, 303], [0, 1, 1, 3], [4, 4, 4, 4]], ids=str)
@pytest.mark.parametrize("behind", [0, 2, 700])
@pytest.mark.parametrize("width", [None, 8])                     # tables of up to 128 tokens are another path
def test_attention(sg, width, behind, starts, bits):
    lens = [100, 64, 2] if width else [900, 64, 2]
    cache, table = made(sg, 31, lens, 16, 2, 64, torch.bfloat16, bits)
    if width:
        table = table[:, :width].contiguous()
    a, b, rows = starts[0], starts[-1], starts[-1] + behind
    q = queries(31, rows, 8, 64, torch.bfloat16)
    n, at, stream = i32(lens), i32(starts), torch.cuda.current_stream().cuda_stream
    work = torch.empty(cache.workspace(8, 2), dtype=torch.uint8, device="cuda")
    for fill in (0, 1):
        o, lse = torch.full_like(q, 7.0), torch.full((8, rows), 7.0, device="cuda")
        desc = [sg.attention._rows(t, "t", q.dtype, 0, 8, 64) for t in (q, o)]
        assert sg.lib().sync_cache_attn(cache.desc, sg.cache._seqs(table, n, at, 0), 8, desc[0], 0.125, 2, desc[1], lse.data_ptr(), fill,
                                        work.data_ptr(), work.numel(), stream) == sg.OK
        for rest, row in ((slice(0, a), slice(0, a)), (slice(b, rows), slice(b, rows))):
            assert bool((o[rest] == (0 if fill else 7)).all()) and bool((lse[:, row] == (-math.inf if fill else 7)).all())
        want = ref.attention(cache, q[a:b], table, lens, [s - a for s in starts], 0.125)
        ref.check((o[a:b], lse[:, a:b]), want)
    new = sg.sync_cache_attn(cache, q, table, n, at, max_new=2, lse=True)
    assert torch.equal(new[0], o) and torch.equal(new[1], lse)


@BITS
def test_append_and_read(sg, bits):
    """The same rows of the other calls."""
    starts, rows, lens = i32([3, 5, 5, 9]), 12, i32([20, 4, 4])
    cache, table = made(sg, 32, [20, 4, 4], 16, 2, 64, torch.bfloat16, bits)
    g = torch.Generator(device="cuda").manual_seed(32)
    q, k, v = (torch.randn((rows, h, 64), generator=g, device="cuda").bfloat16() for h in (8, 2, 2))
    angle = torch.rand((64, 32), generator=g, device="cuda")
    kept = torch.full_like(q, 7.0)
    sg.sync_cache_append(cache, k, v, table, lens, starts, q=q, cos=angle.cos(), sin=angle.sin(), out=kept)
    zero = sg.sync_cache_append(cache, k, v, table, lens, starts, q=q, cos=angle.cos(), sin=angle.sin())
    assert bool((kept[:3] == 7).all()) and bool((kept[9:] == 7).all()) and bool((zero[:3] == 0).all()) and bool((zero[9:] == 0).all())
    assert torch.equal(kept[3:9], zero[3:9])
    given = tuple(torch.full_like(k, 7.0) for _ in range(2))
    sg.sync_cache_read(cache, table, lens, starts, out=given)
    for x, y in zip(given, sg.sync_cache_read(cache, table, lens, starts, rows)):
        assert bool((x[:3] == 7).all()) and bool((x[9:] == 7).all()) and bool((y[:3] == 0).all()) and bool((y[9:] == 0).all())
        assert torch.equal(x[3:9], y[3:9])
    if bits == 16:
        assert torch.equal(y[5:9], v[5:9])          # the third sequence's four tokens, all new
