"""The paged cache on the GPU: rows written to it and read back, against the
format's definition bit for bit, at ragged steps, odd strides, pages in any
order, padding, and places that the table does not have."""
import math

import pytest
import torch

from tests import cache_reference as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def sg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


def i32(x):
    return torch.tensor(x, device="cuda", dtype=torch.int32)


def tables(n, half):
    angle = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))
    return angle.cos().float().cuda(), angle.sin().float().cuda()


def filled(cache, byte=0xC3):
    for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        if t is not None:
            t.view(torch.uint8).fill_(byte)
    return cache


def paged(seed, lens, page, extra=2):
    """(table, pages): the pages of sequences in a random order, -1 past their ends."""
    of = [-(-max(x, 0) // page) for x in lens]
    order = torch.randperm(sum(of) + extra, generator=torch.Generator().manual_seed(seed)).int()
    t = torch.full((len(lens), max(of, default=0) + 1), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(of):
        t[s, :n] = order[at:at + n]
        at += n
    return t.cuda(), sum(of) + extra


def rows(seed, n, heads, dim, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, heads, dim), generator=g, device="cuda")
    return (x * (1 + 3 * (torch.rand((1, heads, dim), generator=g, device="cuda") < 0.03))).to(dtype)   # a few large channels


def expected(sg, cache, before, k, v, q, table, lens, starts, turn):
    """The cache and q_out after an append, by sync_rope and the format."""
    starts = list(range(len(lens) + 1)) if starts is None else starts
    n = k.shape[0]
    pos = torch.full((n,), -1, dtype=torch.int64)
    seq = torch.full((n,), -1, dtype=torch.int64)
    for s in range(len(lens)):
        a, b = starts[s], starts[s + 1]
        pos[a:b] = lens[s] - (b - a) + torch.arange(b - a)
        seq[a:b] = s
    if turn:
        at = dict(turn)
        at.setdefault("positions", pos.int().cuda())
        at.setdefault("interleaved", False)
        exact = [x.cpu() for x in sg.sync_rope(q.float(), k.float(), **at)]
        q_out, kf = exact[0].cuda().to(q.dtype), exact[1].cuda()
    else:
        q_out, kf = q.clone(), k.float()
    mine = seq >= 0
    q_out[~mine.cuda()] = 0
    after = {x: getattr(cache, x).clone() if before is None else before[x].clone() for x in ("k", "v")}
    if cache.bits == 4:
        after.update({x: before[x].clone() for x in ("k_scale", "v_scale")})
    t = table.cpu()
    for r in range(n):
        if not mine[r] or pos[r] < 0 or pos[r] // cache.page >= t.shape[1]:
            continue
        p = int(t[seq[r], pos[r] // cache.page])
        if not 0 <= p < cache.n_pages:
            continue
        o = int(pos[r] % cache.page)
        for x, y in (("k", kf[r]), ("v", v[r].float())):
            if cache.bits == 16:
                after[x][p, :, o] = y.to(k.dtype)
            else:
                after[x][p, :, o], after[x + "_scale"][p, :, o] = ref.encoded(y)
    return q_out, after


def append_and_check(sg, cache, k, v, q, table, lens, starts=None, turn=None, out=None):
    names = ("k", "v") + (("k_scale", "v_scale") if cache.bits == 4 else ())
    before = {x: getattr(cache, x).clone() for x in names}
    want_q, want = expected(sg, cache, before, k, v, q, table, lens, starts, turn)
    got = sg.sync_cache_append(cache, k, v, table, i32(lens), None if starts is None else i32(starts), q=q, out=out, **(turn or {}))
    assert torch.equal(got.view(torch.int16), want_q.view(torch.int16)) or torch.equal(torch.nan_to_num(got), torch.nan_to_num(want_q)) and torch.equal(torch.isnan(got), torch.isnan(want_q))
    for x in names:
        a, b = getattr(cache, x), want[x]
        a, b = (a, b) if a.dtype is torch.uint8 else (a.view(torch.int16), b.view(torch.int16))
        assert torch.equal(a, b), x


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("bits,dim,rotated", [(16, 8, 8), (16, 24, 24), (16, 64, 64), (16, 80, 40), (16, 80, 80), (16, 128, 128), (16, 128, 0), (16, 128, 20),
                                              (4, 32, 32), (4, 64, 64), (4, 64, 22), (4, 96, 96), (4, 96, 48), (4, 128, 128), (4, 128, 64), (4, 128, 0)])
def test_formats(sg, bits, dim, rotated, dtype, interleaved):
    lens, starts, page = [5, 33, 1, 70], [0, 5, 12, 13, 30], 16
    table, pages = paged(dim, lens, page)
    cache = filled(sg.sync_kv_cache(pages, page, 2, dim, dtype, bits=bits))
    k, v, q = (rows(i, 30, h, dim, dtype) for i, h in ((1, 2), (2, 2), (3, 6)))
    cos, sin = tables(100, rotated // 2)
    append_and_check(sg, cache, k, v, q, table, lens, starts, dict(cos=cos, sin=sin, interleaved=interleaved) if rotated else None)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("lens,starts,page", [([1], None, 16), ([17, 16, 300], None, 16), ([64] * 9, None, 32), ([3000], [0, 3000], 64), ([400, 31, 9], [0, 300, 300, 309], 128),
                                              ([1024, 1025], [0, 1024, 2049], 1024), ([], None, 16), ([5] * 70, None, 16)], ids=str)
def test_steps(sg, bits, lens, starts, page):
    table, pages = paged(len(lens), lens, page)
    cache = filled(sg.sync_kv_cache(pages, page, 4, 64, torch.bfloat16, bits=bits))
    n = starts[-1] if starts else len(lens)
    k, v, q = (rows(i, n, h, 64, torch.bfloat16) for i, h in ((4, 4), (5, 4), (6, 4)))
    cos, sin = tables(4000, 32)
    append_and_check(sg, cache, k, v, q, table, lens, starts, dict(cos=cos, sin=sin))


@pytest.mark.parametrize("bits", [16, 4])
def test_padding_and_missing_places(sg, bits):
    """Rows behind the last sequence, sequences without rows, pages that do not
    exist, tokens before the first and past the last page: not written."""
    page, n = 16, 24
    lens, starts = [10, 40, 3, 200, 20], [0, 4, 4, 9, 12, 16]     # the third has more rows than tokens, the fourth is past its pages
    table = i32([[3, -1, -1], [0, 1, 2], [4, 5, 6], [7, 8, 99], [-7, 12, 9]])
    cache = filled(sg.sync_kv_cache(10, page, 2, 64, torch.bfloat16, bits=bits))
    k, v, q = (rows(i, n, h, 64, torch.bfloat16) for i, h in ((7, 2), (8, 2), (9, 8)))
    cos, sin = tables(300, 32)
    append_and_check(sg, cache, k, v, q, table, lens, starts, dict(cos=cos, sin=sin))
    out = torch.full_like(q, 7.0)                                   # given outputs keep what padding rows have
    got = sg.sync_cache_append(cache, k, v, table, i32(lens), i32(starts), q=q, cos=cos, sin=sin, out=out)
    assert got is out and bool((out[16:] == 7.0).all()) and not bool((out[:4] == 7.0).all())


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_strides_in_place_and_axes(sg, bits, shift):
    lens, page, n, heads, kv, dim = [7, 20, 33], 16, 3, 6, 2, 128
    table, pages = paged(3, lens, page)
    wide = torch.full((3, table.shape[1] + 3), -1, dtype=torch.int32, device="cuda")
    wide[:, 1:-2] = table
    cache = filled(sg.sync_kv_cache(pages, page, kv, dim, torch.float16, bits=bits))
    flat = torch.randn((n, (heads + 2 * kv) * dim + 8 + shift), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").half()
    view = flat[:, shift:shift + (heads + 2 * kv) * dim].unflatten(1, (heads + 2 * kv, dim))
    q, k, v = view[:, :heads], view[:, heads:heads + kv], view[:, heads + kv:]
    cos, sin = tables(60, 64)
    turn = dict(cos=cos, sin=sin, positions=i32([[1, 2, 3], [40, 50, 59], [7, 60, 9]]), axes=[0] * 16 + [1] * 24 + [2] * 24)
    append_and_check(sg, cache, k, v, q, wide[:, 1:-2], lens, None, turn)
    append_and_check(sg, cache, k, v, q, wide[:, 1:-2], lens, None, turn, out=q)
    assert sg.sync_cache_append(cache, k, v, table, i32(lens)) is None


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp16"])
def test_values_at_the_ends_of_the_range(sg, dtype):
    """Groups of zeros, of the smallest and largest numbers, with one infinity or
    NaN: the scale's limits."""
    top = torch.finfo(dtype).max
    v = torch.zeros((9, 1, 64), device="cuda", dtype=dtype)
    for r, x in enumerate((0.0, torch.finfo(dtype).tiny, 1e-6, 3e-5, 1e4, top, -top, math.inf, math.nan)):
        v[r, 0, 5] = x
    v[:, 0, 32:] = torch.linspace(-1, 1, 32, device="cuda").to(dtype)
    k = -v
    table, pages = paged(2, [9], 16)
    cache = filled(sg.sync_kv_cache(pages, 16, 1, 64, dtype, bits=4))
    append_and_check(sg, cache, k, v, v.clone(), table, [9], [0, 9])
    kk, vv = sg.sync_cache_read(cache, table, i32([9]), i32([0, 9]), 9)
    assert bool(torch.isnan(vv[7:, 0, :32]).all()) and bool(torch.isnan(kk[7:, 0, :32]).all())
    assert bool(torch.isfinite(vv[:7]).all()) and bool(torch.isfinite(vv[:, :, 32:]).all())
    assert float((vv[4, 0, 5] - 1e4).abs()) <= 1e4 * 2.0 ** -7


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
def test_read(sg, bits, dim):
    lens, page, kv = [1, 0, 50, 300, 16], 16, 3
    table, pages = paged(dim, lens, page)
    cache = sg.sync_kv_cache(pages, page, kv, dim, torch.bfloat16, bits=bits)
    g = torch.Generator(device="cuda").manual_seed(4)
    for t in (cache.k, cache.v):
        t.copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda") if bits == 4 else torch.randn(t.shape, generator=g, device="cuda"))
    if bits == 4:
        for t in (cache.k_scale, cache.v_scale):
            t.copy_(torch.rand(t.shape, generator=g, device="cuda") + 0.1)
    starts = [0, 1, 1, 51, 351, 370]                    # three rows more than the last sequence has, and two of none
    out = tuple(torch.full((372, kv, dim), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    new = sg.sync_cache_read(cache, table, i32(lens), i32(starts), 372)
    sg.sync_cache_read(cache, table, i32(lens), i32(starts), out=out)
    for x, a, b in zip("kv", new, out):
        for s, m in enumerate(lens):
            want = ref.values(cache, x, table[s], m)[0].to(torch.bfloat16)
            assert torch.equal(a[starts[s]:starts[s] + m], want) and torch.equal(b[starts[s]:starts[s] + m], want)
        assert bool((a[367:] == 0).all()) and bool((b[367:370] == 0).all()) and bool((b[370:] == 7).all())
    table[2, 1] = 12345                                  # a page that does not exist
    k, _ = sg.sync_cache_read(cache, table, i32(lens), i32(starts), 372)
    assert bool(torch.isnan(k[17:33]).all()) and torch.equal(k[:17], new[0][:17]) and torch.equal(k[33:], new[0][33:])


def test_offsets_past_32_bits(sg):
    """Pages past 2^32 bytes and 2^31 entries."""
    pages, page, kv, dim = 70_000, 64, 8, 128             # 9.2 GB each
    cache = sg.sync_kv_cache(pages, page, kv, dim, torch.bfloat16)
    table = i32([[69_999, 3], [40_000, 69_000]])
    k, v = rows(1, 130, kv, dim, torch.bfloat16), rows(2, 130, kv, dim, torch.bfloat16)
    sg.sync_cache_append(cache, k, v, table, i32([70, 60]), i32([0, 70, 130]))
    assert torch.equal(cache.k[69_999].transpose(0, 1), k[:64]) and torch.equal(cache.v[40_000, :, :60].transpose(0, 1), v[70:])
    a, b = sg.sync_cache_read(cache, table, i32([70, 60]), i32([0, 70, 130]), 130)
    assert torch.equal(a, k) and torch.equal(b, v)
    q = rows(3, 2, 16, dim, torch.bfloat16)
    want = ref.attention(cache, q, table, [70, 60], None, dim ** -0.5)
    ref.check(sg.sync_cache_attn(cache, q, table, i32([70, 60]), lse=True), want)


def test_refusals(sg):
    bf = torch.bfloat16
    for args in ((4, 8, 2, 64, bf), (4, 16, 0, 64, bf), (4, 16, 2, 60, bf), (4, 16, 2, 64, torch.float32), (-1, 16, 2, 64, bf), (4, 24, 2, 64, bf), (1 << 28, 16, 2, 64, bf),
                 (4, 16.0, 2, 64, bf)):
        with pytest.raises(sg.SyncError):
            sg.sync_kv_cache(*args)
    for bad in (dict(bits=8), dict(bits=4, device="cpu")):
        with pytest.raises(sg.SyncError):
            sg.sync_kv_cache(4, 16, 2, 64, bf, **bad)
    with pytest.raises(sg.SyncError):
        sg.sync_kv_cache(4, 16, 2, 80, bf, bits=4)
    cache = sg.sync_kv_cache(8, 16, 2, 64, bf)
    k, q, table, lens = rows(1, 2, 2, 64, bf), rows(2, 2, 4, 64, bf), i32([[0, 1], [2, 3]]), i32([3, 20])
    cos, sin = tables(30, 32)
    a, r, t = sg.sync_cache_append, sg.sync_cache_read, sg.sync_cache_attn
    for f in (lambda: a(cache, k, k[:1], table, lens), lambda: a(cache, k.half(), k, table, lens), lambda: a(cache, k[:, :1], k, table, lens),
              lambda: a(cache, k, k, table.long(), lens), lambda: a(cache, k, k, table, lens.long()), lambda: a(cache, k, k, table[:1], lens),
              lambda: a(cache, k, k, table[0], lens), lambda: a(cache, k, k, table.cpu(), lens), lambda: a(cache, k, k, table, lens.cpu()),
              lambda: a(cache, k, k, table.T, lens), lambda: a(cache, k, k, table, lens, i32([0, 2])), lambda: a(cache, k, k, table, lens[:1]),
              lambda: a(cache, rows(1, 3, 2, 64, bf), rows(1, 3, 2, 64, bf), table, lens), lambda: a(cache, k, k, table, lens, q=q[:, :3]),
              lambda: a(cache, k, k, table, lens, q=q[:1]), lambda: a(cache, k, k, table, lens, q=q, cos=cos), lambda: a(cache, k, k, table, lens, q=q, out=q[:1].expand(2, 4, 64)),
              lambda: a(cache, k, k, table, lens, cos=tables(30, 33)[0], sin=tables(30, 33)[1]), lambda: r(cache, table, lens, None, 5), lambda: r(cache, table, lens, i32([0, 3, 23])),
              lambda: r(cache, table, lens, i32([0, 3, 23]), -1), lambda: r(cache, table, lens, i32([0, 3, 23]), out=(k, k[:1])), lambda: r(cache, table, lens, i32([0, 3]), 23),
              lambda: t(cache, q[:, :3], table, lens), lambda: t(cache, q[0], table, lens), lambda: t(cache, q.half(), table, lens), lambda: t(cache, q, table, lens, scale=0.0),
              lambda: t(cache, q, table, lens, max_new=0), lambda: t(cache, q[:1], table, lens), lambda: t(cache, q, table, lens, out=q[:1]), lambda: t(cache, q, table, lens, lse=torch.zeros(4, 3, device="cuda")),
              lambda: t(cache, q, table, lens, scale=math.nan), lambda: t(cache, q[..., :32], table, lens)):
        before = sg.kernel_launches()
        with pytest.raises(sg.SyncError) as e:
            f()
        assert e.value.status == sg.ERR_ARG and sg.kernel_launches() == before
    x = q.clone().requires_grad_()
    with pytest.warns(UserWarning, match="sync_cache_attn records nothing"):
        sg.sync_cache_attn(cache, x, table, i32([0, 0]))
