"""Rotation by positions with several axes on the GPU against its definition in
64 bits: types, head sizes, partial and interleaved rotations, axes, strides and
alignments that no wide access fits, its gradient, and its refusals.

Bounds: two products and their sum in 32 bits (2^-24 each of the largest, at most
three roundings), and one rounding to the type."""
import math

import pytest
import torch

from tests import attn_reference as ref

pytestmark = pytest.mark.gpu
U = {**ref.U, torch.float32: 2.0 ** -24}
TINY = {**ref.TINY, torch.float32: 0.0}
DTYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module")
def sg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


def table(n, half):
    angle = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))
    return angle.cos().float().cuda(), angle.sin().float().cuda()


def normal(seed, *shape, dtype):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def turned(x, cos, sin, at, interleaved, way=1.0):
    """at: [rows, half] row of the table for each pair."""
    half = cos.shape[1]
    j = torch.arange(half, device=x.device)
    c, s = cos.double()[at, j][:, None], way * sin.double()[at, j][:, None]
    one = j * 2 if interleaved else j
    two = one + (1 if interleaved else half)
    x = x.double()
    y, size = x.clone(), x.abs()
    y[..., one] = x[..., one] * c - x[..., two] * s
    y[..., two] = x[..., two] * c + x[..., one] * s
    size[..., one] = size[..., two] = x[..., one].abs() + x[..., two].abs()
    return y, size


def near(got, want, size, what):
    t = got.dtype
    tol = U[t] * want.abs() + 3 * 2.0 ** -24 * size + TINY[t]
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), f"{what}: off by {float(off.max()):.3g}"


def run_and_check(sg, q, k, cos, sin, positions, axes, interleaved):
    n, half = q.shape[0], cos.shape[1]
    if positions is None:
        at = torch.arange(n, device="cuda")[:, None].expand(n, half)
    else:
        p = positions.long() if positions.dim() == 2 else positions.long()[None]
        at = p[torch.tensor([0] * half if axes is None else [int(a) for a in axes], device="cuda", dtype=torch.long)].T
    args = dict(positions=positions, axes=axes, interleaved=interleaved)
    for f, way in ((sg.sync_rope, 1.0), (sg.sync_rope_backward, -1.0)):
        got = f(q, k, cos, sin, **args)
        for x, y in zip((q, k), got):
            near(y, *turned(x, cos, sin, at, interleaved, way), f.__name__)
            rest = slice(2 * half, None)
            assert torch.equal(x[..., rest], y[..., rest])           # as it was, bit for bit
    return got


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim,rotated", [(2, 2), (6, 4), (16, 16), (34, 10), (64, 64), (80, 40), (80, 80), (96, 48), (128, 128), (128, 0), (130, 64), (256, 256), (256, 64)])
def test_head_sizes(sg, dim, rotated, dtype, interleaved):
    q, k = normal(1, 37, 5, dim, dtype=dtype), normal(2, 37, 2, dim, dtype=dtype)
    pos = torch.randint(0, 500, (37,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda", dtype=torch.int32)
    run_and_check(sg, q, k, *table(500, rotated // 2), pos, None, interleaved)


@pytest.mark.parametrize("n,heads,kv", [(0, 4, 2), (1, 1, 1), (1, 32, 8), (3, 7, 1), (64, 32, 8), (1000, 4, 4), (5003, 3, 2)])
def test_tokens_heads_and_axes(sg, n, heads, kv):
    q, k = normal(4, n, heads, 128, dtype=torch.bfloat16), normal(5, n, kv, 128, dtype=torch.bfloat16)
    cos, sin = table(max(n, 300), 64)
    run_and_check(sg, q, k, cos, sin, None, None, False)
    g = torch.Generator(device="cuda").manual_seed(6)
    for axes, many in (([0] * 16 + [1] * 24 + [2] * 24, 3), ([j % 4 for j in range(64)], 4), ([1] * 64, 2), (bytes(64), 1)):
        pos = torch.randint(0, 300, (many, n), generator=g, device="cuda", dtype=torch.int32)
        run_and_check(sg, q, k, cos, sin, pos, axes, n % 2 == 1)
    wide = torch.randint(0, 300, (3, n + 5), generator=g, device="cuda", dtype=torch.int32)
    run_and_check(sg, q, k, cos, sin, wide[:, 2:n + 2], torch.tensor([0] * 30 + [2] * 34), False)


@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp16", "fp32"])
def test_strides_and_alignment(sg, dtype, shift):
    n, heads, kv, dim = 129, 6, 2, 128
    flat = normal(7, n, (heads + 2 * kv) * dim + 8 + shift, dtype=dtype)
    view = flat[:, shift:shift + (heads + 2 * kv) * dim].unflatten(1, (heads + 2 * kv, dim))
    pos = torch.arange(n, device="cuda", dtype=torch.int32) * 3
    q, k, (cos, sin) = view[:, :heads], view[:, heads:heads + kv], table(500, 64)
    want = run_and_check(sg, q, k, cos, sin, pos, None, False)
    out = torch.full((heads, n, dim), 7.0, dtype=dtype, device="cuda").transpose(0, 1), torch.full((n, 5, dim), 7.0, dtype=dtype, device="cuda")[:, 1:3]
    sg.sync_rope_backward(q, k, cos, sin, pos, out=out)
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    sg.sync_rope_backward(q, k, cos, sin, pos, out=(q, k))          # in place
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_positions_outside_the_table(sg):
    q, k = normal(8, 6, 4, 64, dtype=torch.bfloat16), normal(9, 6, 2, 64, dtype=torch.bfloat16)
    cos, sin = table(50, 32)
    pos = torch.tensor([[0, -1, 49, 50, 7, 1 << 30], [1, 2, 3, 4, -5, 6]], device="cuda", dtype=torch.int32)
    y = sg.sync_rope(q, k, cos, sin, pos, axes=[0] * 20 + [1] * 12)
    first, second = torch.arange(64, device="cuda") % 32 < 20, torch.arange(64, device="cuda") % 32 >= 20
    for x in y:
        nan = torch.isnan(x).all(1)
        assert torch.equal(nan[:, first].all(1).cpu(), torch.tensor([False, True, False, True, False, True]))
        assert torch.equal(nan[:, second].all(1).cpu(), torch.tensor([False, False, False, False, True, False]))
        assert not bool(torch.isnan(x[[0, 2]]).any())


def test_infinite_entries_stay_with_their_pair(sg):
    q, k = normal(10, 4, 2, 64, dtype=torch.float32), normal(11, 4, 2, 64, dtype=torch.float32)
    cos, sin = table(10, 16)
    clean = sg.sync_rope(q, k, cos, sin)[0]
    q[1, 0, 3], q[2, 1, 40], q[3, 1, 50] = math.inf, math.nan, -math.inf
    y = sg.sync_rope(q, k, cos, sin)[0]
    same = torch.ones_like(y, dtype=torch.bool)
    same[1, 0, 3] = same[1, 0, 19] = same[2, 1, 40] = same[3, 1, 50] = False
    assert torch.equal(y[same], clean[same]) and float(y[3, 1, 50]) == -math.inf


def test_gradient_against_differences(sg):
    """A rotation is linear: its product with a direction is the gradient's."""
    q, k = normal(12, 30, 4, 64, dtype=torch.float32), normal(13, 30, 2, 64, dtype=torch.float32)
    dq, dk = normal(14, 30, 4, 64, dtype=torch.float32), normal(15, 30, 2, 64, dtype=torch.float32)
    cos, sin = table(40, 32)
    y, g = sg.sync_rope(q, k, cos, sin), sg.sync_rope_backward(dq, dk, cos, sin)
    for x, t, d, e in ((q, y[0], dq, g[0]), (k, y[1], dk, g[1])):
        a, b = (t.double() * d.double()).sum(), (x.double() * e.double()).sum()
        assert abs(float(a - b)) <= 4 * 2.0 ** -24 * float((t.double().abs() * d.double().abs()).sum() * 2 + (x.double().abs() * e.double().abs()).sum() * 2)


def test_offsets_past_32_bits(sg):
    """A tensor whose rows lie more than 2^31 entries apart."""
    base = torch.zeros((2, 1_100_000_000), dtype=torch.bfloat16, device="cuda")
    q, k = base[:, :256].unflatten(1, (4, 64)), base[:, 1_099_999_744:].unflatten(1, (4, 64))
    q.copy_(normal(16, 2, 4, 64, dtype=torch.bfloat16))
    k.copy_(normal(17, 2, 4, 64, dtype=torch.bfloat16))
    run_and_check(sg, q, k, *table(9, 32), torch.tensor([3, 8], device="cuda", dtype=torch.int32), None, False)


def test_graph_and_stream(sg):
    q, k = normal(18, 70, 4, 128, dtype=torch.bfloat16), normal(19, 70, 2, 128, dtype=torch.bfloat16)
    cos, sin = table(300, 64)
    pos = torch.arange(70, device="cuda", dtype=torch.int32)
    out, graph = (torch.empty_like(q), torch.empty_like(k)), torch.cuda.CUDAGraph()
    sg.sync_rope(q, k, cos, sin, pos, out=out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sg.sync_rope(q, k, cos, sin, pos, out=out)
    pos += 100                                                        # a replay follows what the positions are
    graph.replay()
    want = sg.sync_rope(q, k, cos, sin, pos)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    other = sg.sync_rope(q, k, cos, sin, pos, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(x, y) and torch.equal(x, z) for x, y, z in zip(want, out, other))


def test_refusals(sg):
    q, k, (cos, sin) = normal(20, 5, 4, 64, dtype=torch.bfloat16), normal(21, 5, 2, 64, dtype=torch.bfloat16), table(9, 32)
    pos = torch.zeros(5, device="cuda", dtype=torch.int32)
    bad = [lambda: sg.sync_rope(q[:4], k, cos, sin), lambda: sg.sync_rope(q, k.half(), cos, sin), lambda: sg.sync_rope(q.cpu(), k, cos, sin),
           lambda: sg.sync_rope(q, k, cos.double(), sin.double()), lambda: sg.sync_rope(q, k, cos, sin[:5]), lambda: sg.sync_rope(q, k, cos[0], sin[0]),
           lambda: sg.sync_rope(q, k, *table(9, 33)), lambda: sg.sync_rope(q, k, cos, sin, pos.long()), lambda: sg.sync_rope(q, k, cos, sin, pos[:4]),
           lambda: sg.sync_rope(q, k, cos, sin, pos.cpu()), lambda: sg.sync_rope(q, k, cos, sin, torch.zeros(2, 5, device="cuda", dtype=torch.int32)),
           lambda: sg.sync_rope(q, k, cos, sin, torch.zeros(5, 5, device="cuda", dtype=torch.int32), axes=[0] * 32),
           lambda: sg.sync_rope(q, k, cos, sin, pos, axes=[0] * 31), lambda: sg.sync_rope(q, k, cos, sin, pos, axes=[0] * 31 + [1]),
           lambda: sg.sync_rope(q, k, cos, sin, pos, axes=[0] * 31 + [-1]), lambda: sg.sync_rope(q, k, cos, sin, axes=[1] * 32),
           lambda: sg.sync_rope(q, k, cos, sin, torch.zeros(5, 2, device="cuda", dtype=torch.int32).T, axes=[0] * 32),
           lambda: sg.sync_rope(q.int(), k.int(), cos, sin), lambda: sg.sync_rope(q, k, cos, sin, out=(q, q)),
           lambda: sg.sync_rope(q, k, cos, sin, out=(q[:1].expand(5, 4, 64), k)), lambda: sg.sync_rope(q.transpose(1, 2), k, cos, sin)]
    for f in bad:
        before = sg.kernel_launches()
        with pytest.raises(sg.SyncError) as e:
            f()
        assert e.value.status == sg.ERR_ARG and sg.kernel_launches() == before
    x = q.float().requires_grad_()
    with pytest.warns(UserWarning, match="sync_rope records nothing"):
        sg.sync_rope(x, k.float(), cos, sin)


def test_in_an_autograd_function(sg):
    """On the backward pass's thread, with two uses of the same leaf."""
    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, cos, sin, pos):
            ctx.save_for_backward(cos, sin, pos)
            return sg.sync_rope(q, k, cos, sin, pos)

        @staticmethod
        def backward(ctx, dq, dk):
            return (*sg.sync_rope_backward(dq.contiguous(), dk.contiguous(), *ctx.saved_tensors), None, None, None)

    g = torch.Generator(device="cuda").manual_seed(4)
    q, k = (torch.randn(50, h, 64, generator=g, device="cuda").requires_grad_() for h in (4, 2))
    angle = torch.randn(70, 32, generator=g, device="cuda")
    pos = torch.randint(0, 70, (50,), generator=g, device="cuda", dtype=torch.int32)
    weights = [torch.randn(t.shape, generator=g, device="cuda") for t in (q, k)]
    a, b = Turn.apply(q, k, angle.cos(), angle.sin(), pos)
    ((a * weights[0]).sum() + (b * weights[1]).sum() + (q * 2).sum()).backward()
    dq, dk = sg.sync_rope_backward(*weights, angle.cos(), angle.sin(), pos)
    assert torch.equal(q.grad, dq + 2) and torch.equal(k.grad, dk)
