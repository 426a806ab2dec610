"""Attention over the paged cache on the GPU against its definition in 64 bits
(cache_reference.py, which derives the bounds): both formats, types, head
layouts and sizes, page sizes, lengths from none on, several new tokens,
padding, places that do not exist, what lies past a sequence's end, long and
many sequences, graphs and streams."""
import math

import pytest
import torch

from tests import cache_reference as ref
from tests.test_gpu_cache import i32, paged

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


def made(sg, seed, lens, page, kv, dim, dtype, bits, spread=0.3):
    """A cache with random rows everywhere, and the table of its sequences."""
    table, pages = paged(seed, lens, page)
    cache = sg.sync_kv_cache(pages, page, kv, dim, dtype, bits=bits)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for t in (cache.k, cache.v):
        t.copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda") if bits == 4 else torch.randn(t.shape, generator=g, device="cuda"))
    if bits == 4:
        for t in (cache.k_scale, cache.v_scale):
            t.copy_((0.2 * torch.exp(spread * torch.randn(t.shape, generator=g, device="cuda"))).clamp(max=65504.0))   # the format's largest
    return cache, table


def queries(seed, n, heads, dim, dtype, gain=1.5):
    return (torch.randn((n, heads, dim), generator=torch.Generator(device="cuda").manual_seed(seed + 99), device="cuda") * gain).to(dtype)


def run_and_check(sg, lens, heads, kv, dim, dtype, bits, page=16, starts=None, max_new=1, scale=None, gain=1.5, seed=1, spread=0.3):
    cache, table = made(sg, seed, lens, page, kv, dim, dtype, bits, spread)
    q = queries(seed, starts[-1] if starts else len(lens), heads, dim, dtype, gain)
    args = (cache, q, table, i32(lens), None if starts is None else i32(starts))
    got = sg.sync_cache_attn(*args, max_new=max_new, scale=scale, lse=True)
    ref.check(got, ref.attention(cache, q, table, lens, starts, scale or dim ** -0.5))
    assert torch.equal(sg.sync_cache_attn(*args, max_new=max_new, scale=scale), got[0])


BITS = pytest.mark.parametrize("bits", [16, 4])
DTYPE = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])


@BITS
@DTYPE
@pytest.mark.parametrize("lens", [[1], [16], [17, 2], [64, 63, 65], [0, 5, 0], [128, 1, 129, 1000], [3000], [700] * 20], ids=str)
def test_lengths(sg, lens, dtype, bits):
    run_and_check(sg, lens, 8, 2, 128, dtype, bits)
    run_and_check(sg, lens, 8, 2, 64, dtype, bits, page=64)


@BITS
@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (6, 2), (5, 1), (8, 1), (16, 2), (16, 1), (20, 1), (40, 2), (65, 5)], ids=str)
def test_head_layouts(sg, heads, kv, bits):
    run_and_check(sg, [150, 1, 333], heads, kv, 128, torch.bfloat16, bits)
    run_and_check(sg, [150, 0, 333], heads, kv, 64, torch.float16, bits)


@DTYPE
@pytest.mark.parametrize("bits,dim", [(16, x) for x in (8, 16, 24, 40, 56, 72, 80, 96, 104, 120)] + [(4, 32), (4, 96)])
def test_head_sizes(sg, bits, dim, dtype):
    run_and_check(sg, [77, 200], 4, 2, dim, dtype, bits)
    run_and_check(sg, [77, 200], 12, 1, dim, dtype, bits, page=32)


@BITS
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 512, 1024])
def test_pages(sg, page, bits):
    run_and_check(sg, [2000, 31, 513], 8, 2, 128, torch.bfloat16, bits, page=page)


@BITS
@pytest.mark.parametrize("tokens,max_new", [([1, 1, 1], 1), ([5, 5, 5], 5), ([3, 0, 7], 7), ([9, 1, 2], 9), ([40, 1, 17], 40), ([9, 1, 2], 1)], ids=str)
def test_several_new_tokens(sg, tokens, max_new, bits):
    """Each sees the cache up to itself; max_new chooses a tile, no more."""
    starts = [sum(tokens[:i]) for i in range(4)]
    for heads, kv, dim, dtype in ((8, 2, 128, torch.bfloat16), (5, 1, 64, torch.float16), (3, 3, 64, torch.bfloat16)):
        run_and_check(sg, [100, 700, 40], heads, kv, dim, dtype, bits, starts=starts, max_new=max_new)


@BITS
def test_more_rows_than_tokens(sg, bits):
    """The first rows of such a sequence see nothing: zeros."""
    run_and_check(sg, [3, 0, 5], 4, 2, 64, torch.bfloat16, bits, starts=[0, 7, 9, 14], max_new=7)


@BITS
@DTYPE
@pytest.mark.parametrize("gain", [0.0, 12.0, 60.0])
def test_flat_and_peaked_rows(sg, gain, dtype, bits):
    run_and_check(sg, [900, 300], 8, 2, 128, dtype, bits, gain=gain)
    run_and_check(sg, [900, 300], 8, 2, 128, dtype, bits, scale=0.01 if gain else 3.0, gain=gain or 1.0)


@BITS
def test_long_and_many(sg, bits):
    run_and_check(sg, [20011], 8, 2, 128, torch.bfloat16, bits, page=64)
    run_and_check(sg, [9000, 1, 5000, 64], 16, 2, 64, torch.float16, bits, page=32)
    run_and_check(sg, [(i * 37) % 90 for i in range(700)], 2, 1, 64, torch.bfloat16, bits)


def test_scales_of_very_different_size(sg):
    """Groups whose scales differ by powers of ten, larger ones later."""
    for spread in (3.0, 5.0):
        run_and_check(sg, [400, 70], 4, 2, 128, torch.bfloat16, 4, spread=spread, scale=1e-3)
    cache, table = made(sg, 3, [600], 16, 1, 64, torch.bfloat16, 4)
    at = torch.arange(cache.v_scale.shape[0], device="cuda").view(-1, 1, 1, 1)
    for big, small in ((60000.0, 1e-3), (1e-6, 1e-7), (1.0, 0.0)):
        cache.v_scale.copy_(torch.where(at % 3 == 0, big, small).expand_as(cache.v_scale))
        q = queries(3, 1, 4, 64, torch.bfloat16)
        ref.check(sg.sync_cache_attn(cache, q, table, i32([600]), lse=True), ref.attention(cache, q, table, [600], None, 64 ** -0.5))


def test_queries_of_any_size(sg):
    """4 bits scale queries to float16's range: large and small ones, heads with
    entries of both, a head of zeros."""
    cache, table = made(sg, 4, [300], 16, 2, 128, torch.bfloat16, 4)
    q = queries(4, 1, 8, 128, torch.bfloat16)
    q[0, 0] *= 1e30
    q[0, 1] *= 1e-30
    q[0, 2, ::2] *= 1e5
    q[0, 3] = 0
    q[0, 4, 1:] = 0
    for scale in (1e-31, 0.1, 1e3):
        keep = torch.tensor([i for i in range(8) if (scale < 1e-30 or i != 0) and (scale < 1 or i != 2)], device="cuda")
        o, lse = sg.sync_cache_attn(cache, q, table, i32([300]), scale=scale, lse=True)
        want = ref.attention(cache, q, table, [300], None, scale)
        mine = {x: t[:, keep] if x.startswith("o") else t[keep] for x, t in want.items()}
        ref.check((o[:, keep], lse[keep]), mine)


@BITS
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_no_row_sees_reaches_none(sg, bad, bits):
    """Past the ends of the sequences, and in pages of others, anything."""
    lens, page = [70, 33, 16, 130], 64
    cache, table = made(sg, 5, lens, page, 2, 64, torch.bfloat16, bits)
    q = queries(5, 4, 8, 64, torch.bfloat16)
    clean = sg.sync_cache_attn(cache, q, table, i32(lens), lse=True)
    seen = torch.zeros((cache.n_pages, page), dtype=torch.bool, device="cuda")
    for s, n in enumerate(lens):
        if s != 1:
            seen[ref.places(table[s], page, n)] = True
    for t in (cache.k, cache.v) if bits == 16 else (cache.k_scale, cache.v_scale):
        t.transpose(1, 2)[~seen] = bad
    dirty = sg.sync_cache_attn(cache, q, table, i32(lens), lse=True)
    for s in (0, 2, 3):
        assert torch.equal(clean[0][s], dirty[0][s]) and torch.equal(clean[1][:, s], dirty[1][:, s])


@BITS
def test_padding_and_missing_pages(sg, bits):
    lens, starts = [200, 90, 100, 5], [0, 2, 5, 6, 8]
    cache, table = made(sg, 6, lens, 16, 2, 64, torch.bfloat16, bits)
    q = queries(6, 11, 8, 64, torch.bfloat16)
    want = ref.attention(cache, q, table, lens, starts, 0.125)
    got = sg.sync_cache_attn(cache, q, table, i32(lens), i32(starts), max_new=3, lse=True)
    ref.check(got, want)
    assert bool((got[0][8:] == 0).all()) and bool((got[1][:, 8:] == -math.inf).all())
    out, lse = torch.full_like(q, 7.0), torch.full((8, 11), 7.0, device="cuda")
    sg.sync_cache_attn(cache, q, table, i32(lens), i32(starts), max_new=3, out=out, lse=lse)
    assert torch.equal(out[:8], got[0][:8]) and bool((out[8:] == 7).all()) and bool((lse[:, 8:] == 7).all())
    broken = table.clone()
    broken[0, 7], broken[3, 0] = cache.n_pages, -1
    lens[2] = 16 * table.shape[1] + 1                    # more tokens than its pages hold
    o, lse = sg.sync_cache_attn(cache, q, broken, i32(lens), i32(starts), max_new=3, lse=True)
    for a, b, bad in ((0, 2, True), (2, 5, False), (5, 6, True), (6, 8, True)):
        assert bool(torch.isnan(o[a:b]).all()) == bad and bool(torch.isnan(lse[:, a:b]).all()) == bad
        assert bad or torch.equal(o[a:b], got[0][a:b])


@BITS
def test_shared_pages(sg, bits):
    """Sequences with a common beginning read the same pages."""
    cache, table = made(sg, 7, [200, 200], 16, 2, 128, torch.bfloat16, bits)
    table[1, :8] = table[0, :8]
    q = queries(7, 2, 8, 128, torch.bfloat16)
    ref.check(sg.sync_cache_attn(cache, q, table, i32([200, 190]), lse=True), ref.attention(cache, q, table, [200, 190], None, 128 ** -0.5))


@BITS
def test_strided_tensors(sg, bits):
    cache, table = made(sg, 8, [300, 40], 32, 2, 64, torch.bfloat16, bits)
    wide = queries(8, 2, 12, 64, torch.bfloat16)
    q, out = wide[:, 2:10], torch.full((8, 2, 72), 7.0, device="cuda", dtype=torch.bfloat16).transpose(0, 1)[..., :64]
    sg.sync_cache_attn(cache, q, table, i32([300, 40]), out=out)
    assert torch.equal(out, sg.sync_cache_attn(cache, q.contiguous(), table, i32([300, 40])))


@BITS
def test_graphs_streams_and_lengths_that_grow(sg, bits):
    """A captured step follows its lengths; two graphs and a stream of their own
    do not share a workspace."""
    lens = [500, 3000, 64, 1]
    cache, table = made(sg, 9, [x + 64 for x in lens], 16, 2, 128, torch.bfloat16, bits)
    q, n = queries(9, 4, 8, 128, torch.bfloat16), i32(lens)
    outs, graphs = [torch.empty_like(q) for _ in range(2)], [torch.cuda.CUDAGraph() for _ in range(2)]
    sg.sync_cache_attn(cache, q, table, n)
    torch.cuda.synchronize()
    for g, o in zip(graphs, outs):
        with torch.cuda.graph(g):
            sg.sync_cache_attn(cache, q, table, n, out=o)
    sides = [torch.cuda.Stream() for _ in range(2)]
    for step in range(5):
        n += 1 if step % 2 else 11
        torch.cuda.synchronize()
        for g, s in zip(graphs, sides):
            with torch.cuda.stream(s):
                g.replay()
        other = sg.sync_cache_attn(cache, q, table, n, stream=sides[0])
        torch.cuda.synchronize()
        want = sg.sync_cache_attn(cache, q, table, n)
        assert all(torch.equal(want, x) for x in outs + [other])
        ref.check((want, None), ref.attention(cache, q, table, n.tolist(), None, 128 ** -0.5))


def test_nothing_to_do(sg):
    cache = sg.sync_kv_cache(0, 16, 2, 64, torch.bfloat16)
    e = torch.empty((0, 4, 64), device="cuda", dtype=torch.bfloat16)
    t = torch.empty((0, 0), device="cuda", dtype=torch.int32)
    assert sg.sync_cache_attn(cache, e, t, i32([])).shape == (0, 4, 64)
    o = sg.sync_cache_attn(cache, torch.ones((2, 4, 64), device="cuda", dtype=torch.bfloat16), torch.empty((2, 0), device="cuda", dtype=torch.int32), i32([0, 0]))
    assert bool((o == 0).all())


@BITS
def test_short_tables_and_small_workspaces(sg, bits):
    """Sequences of up to 128 tokens by way of short tables take no workspace; others
    are refused one that is too small."""
    lens = [128, 0, 1, 77, 64] * 30
    run_and_check(sg, lens, 8, 2, 128, torch.bfloat16, bits, page=128)
    run_and_check(sg, [16, 0, 3, 100], 10, 2, 64, torch.float16, bits, page=64, starts=[0, 3, 4, 4, 9], max_new=5)
    cache, table = made(sg, 10, [200], 16, 2, 64, torch.bfloat16, bits)
    q, n = queries(10, 1, 8, 64, torch.bfloat16), i32([200])
    C, rows = sg.cache, sg.attention._rows(q, "q", q.dtype, 0, 8, 64)
    work = torch.empty(cache.workspace(8, 1), dtype=torch.uint8, device="cuda")
    for size, status in ((work.numel() - 1, sg.ERR_ARG), (work.numel(), sg.OK)):
        assert sg.lib().sync_cache_attn(cache.desc, C._seqs(table, n, None, 0), 8, rows, 0.1, 1, rows, None, 0, work.data_ptr(), size, None) == status
    torch.cuda.synchronize()


@BITS
def test_run_of_a_prompt_and_its_answer(sg, bits):
    """A prompt appended in pieces, read back for the packed attention of the
    next piece, then decoded token by token: as attention over all of it."""
    heads, kv, dim, dtype, page = 8, 2, 64, torch.bfloat16, 16
    pieces = [[40, 17], [30, 0], [1, 1], [1, 1]]
    g = torch.Generator(device="cuda").manual_seed(11)
    cache, lens = sg.sync_kv_cache(20, page, kv, dim, dtype, bits=bits), [0, 0]
    table = torch.randperm(20, generator=torch.Generator().manual_seed(1)).int().view(2, 10).cuda()
    angle = torch.arange(200, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(32, device="cuda", dtype=torch.float64) / 32)
    cos, sin = angle.cos().float(), angle.sin().float()
    for new in pieces:
        lens = [x + y for x, y in zip(lens, new)]
        starts = i32([0, new[0], sum(new)])
        q, k, v = (torch.randn((sum(new), h, dim), generator=g, device="cuda").to(dtype) for h in (heads, kv, kv))
        q = sg.sync_cache_append(cache, k, v, table, i32(lens), starts, q=q, cos=cos, sin=sin)
        want = ref.attention(cache, q, table, lens, [0, new[0], sum(new)], dim ** -0.5)
        ref.check(sg.sync_cache_attn(cache, q, table, i32(lens), starts, max_new=max(new), lse=True), want)
        kk, vv = sg.sync_cache_read(cache, table, i32(lens), i32([0, lens[0], sum(lens)]), sum(lens))
        plan = sg.sync_attn_plan(new, lens, heads, kv, dim, dtype)
        o = sg.sync_attn_forward(plan, q, kk, vv)
        # the values read back are rounded once more to 16 bits in 4-bit caches, scores by twice that of their products
        tol = want["o_tol"] + (0 if bits == 16 else 2.0 ** -6) * want["o"].abs().amax() + 2.0 ** -8 * want["o"].abs()
        assert bool(((o.double() - want["o"]).abs() <= tol).all())
        plan.close()


@BITS
def test_slots_without_rows(sg, bits):
    """A step of a server whose slots are mostly idle: they have no rows, whatever their lengths say."""
    lens = [0] * 90 + [40] * 200 + [333] + [9000] * 500 + [70, 1] + [0] * 300 + [129]
    tokens = [0] * 290 + [2] + [0] * 500 + [1, 1] + [0] * 300 + [3]
    starts = [sum(tokens[:i]) for i in range(len(tokens) + 1)]
    busy = [s for s, n in enumerate(tokens) if n]
    cache, few = made(sg, 9, [lens[s] for s in busy], 16, 2, 64, torch.bfloat16, bits)
    table = torch.full((len(lens), few.shape[1]), -1, dtype=torch.int32, device="cuda")
    table[busy] = few
    q = queries(9, 9, 8, 64, torch.bfloat16)
    got = sg.sync_cache_attn(cache, q, table, i32(lens), i32(starts), max_new=3, lse=True)
    some = [lens[s] for s in busy], [sum(tokens[s] for s in busy[:i]) for i in range(len(busy) + 1)]
    ref.check((got[0][:7], got[1][:, :7]), ref.attention(cache, q[:7], few, *some, 0.125))
    assert bool((got[0][7:] == 0).all())


@BITS
def test_pages_past_32_bits(sg, bits):
    """The same tokens on the last pages of a cache of more than 4 GiB a tensor, and in a small one."""
    page, kv, dim, lens = 1024, 8, 128, [1500, 3, 1025]
    n = 2100 if bits == 16 else 8300
    small, table = made(sg, 11, lens, page, kv, dim, torch.bfloat16, bits)
    large = sg.sync_kv_cache(n, page, kv, dim, torch.bfloat16, bits=bits)
    assert large.k.numel() * large.k.element_size() > 1 << 32
    for name in ("k", "v", "k_scale", "v_scale"):
        t = getattr(small, name)
        if t is not None:
            getattr(large, name)[n - small.n_pages:] = t
    q = queries(11, 3, 32, dim, torch.bfloat16)
    want = sg.sync_cache_attn(small, q, table, i32(lens), lse=True)
    got = sg.sync_cache_attn(large, q, torch.where(table < 0, table, table + n - small.n_pages), i32(lens), lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@BITS
def test_two_calls_at_once(sg, bits):
    """Calls on two streams, each with the workspace that it allocates."""
    cache, table = made(sg, 12, [5000, 20, 3000], 64, 4, 128, torch.bfloat16, bits)
    lens, some = i32([5000, 20, 3000]), i32([4000, 0, 2999])
    q = queries(12, 3, 16, 128, torch.bfloat16)
    want = sg.sync_cache_attn(cache, q, table, lens), sg.sync_cache_attn(cache, q, table, some)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [[sg.sync_cache_attn(cache, q, table, n, stream=s) for s, n in zip(streams, (lens, some))] for _ in range(20)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[0]) and torch.equal(b, want[1]) for a, b in got)


@BITS
def test_on_a_thread_of_its_own(sg, bits):
    """A thread that has made no call of the runtime yet."""
    import threading
    cache, table = made(sg, 13, [700, 40], 32, 2, 64, torch.float16, bits)
    q, lens, got = queries(13, 2, 4, 64, torch.float16), i32([700, 40]), []
    want = sg.sync_cache_attn(cache, q, table, lens, lse=True)
    t = threading.Thread(target=lambda: got.extend(sg.sync_cache_attn(cache, q, table, lens, lse=True)))
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
