"""The attention over the paged cache on workspaces as a caller of the C entry may
place them: at any multiple of 16 bytes, of exactly the size asked for, with
whatever the memory held before."""
import pytest
import torch

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
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("heads,max_new", [(8, 1), (16, 1), (16, 3)], ids=str)
@pytest.mark.parametrize("shift", [0, 16, 32, 48, 240])
def test_at_any_multiple_of_16_bytes(sg, shift, heads, max_new, dim, bits):
    lens = [5000, 1, 3000, 700]                    # cut between warps and between blocks
    cache, table = made(sg, 21, lens, 64, 2, dim, torch.bfloat16, bits)
    starts = [max_new * s for s in range(5)]
    q = queries(21, starts[-1], heads, dim, torch.bfloat16)
    want = sg.sync_cache_attn(cache, q, table, i32(lens), i32(starts), max_new=max_new)
    size = cache.workspace(heads, max_new)
    memory = torch.full((size + 512,), 0x7f, dtype=torch.uint8, device="cuda")
    first = -memory.data_ptr() % 256 + shift
    o = torch.zeros_like(q)
    n, at = i32(lens), i32(starts)
    rows = [sg.attention._rows(t, "t", q.dtype, 0, heads, dim) for t in (q, o)]
    assert sg.lib().sync_cache_attn(cache.desc, sg.cache._seqs(table, n, at, 0), heads, rows[0], dim ** -0.5, max_new, rows[1], None, 0,
                                    memory.data_ptr() + first, size, torch.cuda.current_stream().cuda_stream) == sg.OK
    assert torch.equal(o, want)
    assert bool((memory[:first] == 0x7f).all()) and bool((memory[first + size:] == 0x7f).all())
