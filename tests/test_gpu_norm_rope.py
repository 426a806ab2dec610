"""Head norms with the position rotation on the GPU against their definition in
64 bits: types, head sizes, partial and interleaved rotations, strides and
alignments that no wide access fits, their gradient, and their refusals.

Bounds: everything is computed in 32 bits and rounded once to the type (u of
attn_reference, 2^-24 for float32); the 32-bit part is a sum of at most 256
squares and a few products, below 2^-18 relative to the largest entry that
enters a result.  A weight's gradient sums n products in 32 bits in a tree:
below 2^-24 (20 + log2 n) times the sum of their sizes."""
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


def table(n, rotated, device="cuda"):
    half = rotated // 2
    angle = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))
    return angle.cos().float().to(device), angle.sin().float().to(device)


def made(seed, n, heads, kv, dim, dtype, weights=True):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*s, std=1.0):
        return (torch.randn(s, generator=g, device="cuda") * std).to(dtype)
    w = [(1 + 0.2 * torch.randn(dim, generator=g, device="cuda")).to(dtype) if weights else None for _ in range(2)]
    pos = torch.randint(0, 500, (n,), generator=g, device="cuda", dtype=torch.int32)
    return normal(n, heads, dim, std=1.7), normal(n, kv, dim, std=0.4), normal(n, heads, dim), normal(n, kv, dim), w, pos


def near(got, want, dtype, scale, name):
    tol = U[dtype] * want.abs() + 2.0 ** -18 * scale + TINY[dtype]
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), f"{name}: off by {float(off.max()):.3g}"


def run_and_check(sg, q, k, gq, gk, w, cos, sin, pos, interleaved, eps=1e-6, positions=True):
    dtype = q.dtype
    at = pos if positions else torch.arange(q.shape[0], device="cuda")
    args = (w[0], w[1], cos, sin, pos if positions else None)
    out = sg.sync_qk_norm_rope(q, k, *args, eps=eps, interleaved=interleaved)
    for x, y, wi, name in ((q, out[0], w[0], "q"), (k, out[1], w[1], "k")):
        want = ref.norm_rope(x, wi, cos, sin, at, eps, interleaved)
        near(y, want, dtype, want.abs().amax(-1, keepdim=True), name)
    got = sg.sync_qk_norm_rope_backward(q, k, gq, gk, *args, eps=eps, interleaved=interleaved)
    for x, d, wi, dx, dw, name in ((q, gq, w[0], got[0], got[2], "q"), (k, gk, w[1], got[1], got[3], "k")):
        want, want_w, sizes = ref.norm_rope(x, wi, cos, sin, at, eps, interleaved, d)
        r = (x.double().square().mean(-1, keepdim=True) + eps).rsqrt()
        scale = r * (d.double().abs().amax(-1, keepdim=True) * 2 * (1 if wi is None else float(wi.abs().max())))
        near(dx, want, dtype, 4 * scale, "d" + name)
        if wi is None:
            assert dw is None
            continue
        n = max(2, x.shape[0] * x.shape[1])
        tol = 2.0 ** -24 * (20 + math.log2(n)) * sizes + U[dtype] * want_w.abs() + TINY[dtype]
        assert bool(((dw.double() - want_w).abs() <= tol).all()), f"dw{name}: off by {float((dw.double() - want_w).abs().max()):.3g}"
    again = sg.sync_qk_norm_rope_backward(q, k, gq, gk, *args, eps=eps, interleaved=interleaved)
    assert all(x is y or torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim,rotated", [(2, 2), (6, 4), (16, 16), (34, 10), (64, 64), (80, 40), (80, 80), (96, 48), (128, 128), (128, 0), (130, 64), (256, 256), (256, 64)])
def test_head_sizes(sg, dim, rotated, dtype, interleaved):
    q, k, gq, gk, w, pos = made(dim, 37, 5, 2, dim, dtype)
    cos, sin = table(500, rotated)
    run_and_check(sg, q, k, gq, gk, w, cos, sin, pos, interleaved)


@pytest.mark.parametrize("n,heads,kv", [(1, 1, 1), (1, 32, 8), (3, 7, 1), (64, 32, 8), (1000, 4, 4), (5003, 3, 2)])
def test_tokens_and_heads(sg, n, heads, kv):
    q, k, gq, gk, w, pos = made(n, n, heads, kv, 128, torch.bfloat16)
    cos, sin = table(max(n, 500), 128)
    run_and_check(sg, q, k, gq, gk, w, cos, sin, pos, False)
    run_and_check(sg, q, k, gq, gk, w, cos, sin, pos, False, positions=False)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp16", "fp32"])
def test_without_weights_and_zero_rows(sg, dtype):
    q, k, gq, gk, w, pos = made(4, 50, 4, 2, 64, dtype, weights=False)
    q[7] = 0
    k[9] = 0
    run_and_check(sg, q, k, gq, gk, w, *table(500, 64), pos, False, eps=1e-3)


@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp16", "fp32"])
def test_strides_and_alignment(sg, dtype, shift):
    """Views of a fused projection, shifted off every wide boundary."""
    n, heads, kv, dim = 129, 6, 2, 128
    g = torch.Generator(device="cuda").manual_seed(2)
    flat = torch.randn((2, n, (heads + 2 * kv) * dim + 8 + shift), generator=g, device="cuda").to(dtype)
    view = flat[:, :, shift:shift + (heads + 2 * kv) * dim].unflatten(2, (heads + 2 * kv, dim))
    w = [torch.ones(dim, device="cuda", dtype=dtype) * 1.1, torch.ones(dim + 1, device="cuda", dtype=dtype)[1:]]
    pos = torch.arange(n, device="cuda", dtype=torch.int32) * 3
    run_and_check(sg, view[0, :, :heads], view[0, :, heads:heads + kv], view[1, :, :heads], view[1, :, heads:heads + kv], w, *table(500, dim), pos, False)


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
def test_in_place(sg, interleaved):
    q, k, gq, gk, w, pos = made(5, 300, 8, 2, 128, torch.bfloat16)
    cos, sin = table(500, 128)
    a = (w[0], w[1], cos, sin, pos)
    want = sg.sync_qk_norm_rope(q, k, *a, interleaved=interleaved)
    grad = sg.sync_qk_norm_rope_backward(q, k, gq, gk, *a, interleaved=interleaved)
    sg.sync_qk_norm_rope_backward(q, k, gq, gk, *a, interleaved=interleaved, out=(gq, gk))
    assert torch.equal(gq, grad[0]) and torch.equal(gk, grad[1])
    sg.sync_qk_norm_rope(q, k, *a, interleaved=interleaved, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_positions_outside_the_table(sg):
    q, k, gq, gk, w, pos = made(6, 20, 4, 2, 64, torch.bfloat16)
    cos, sin = table(100, 64)
    pos = pos % 100
    good = sg.sync_qk_norm_rope(q, k, w[0], w[1], cos, sin, pos)
    pos[3], pos[11] = 100, -1
    for x, y in zip(sg.sync_qk_norm_rope(q, k, w[0], w[1], cos, sin, pos), good):
        assert bool(torch.isnan(x[[3, 11]]).all())
        rest = [i for i in range(20) if i not in (3, 11)]
        assert torch.equal(x[rest], y[rest])


def test_gradient_against_differences(sg):
    q, k, gq, gk, w, pos = made(7, 30, 4, 2, 64, torch.float32)
    cos, sin = table(500, 48)
    got = sg.sync_qk_norm_rope_backward(q, k, gq, gk, w[0], w[1], cos, sin, pos)

    def loss(x, wi, d):
        return float((ref.norm_rope(x, wi, cos, sin, pos, 1e-6, False) * d.double()).sum())
    g = torch.Generator(device="cuda").manual_seed(8)
    for x, d, wi, dx, dw in ((q, gq, w[0], got[0], got[2]), (k, gk, w[1], got[1], got[3])):
        x, wi, h = x.double(), wi.double(), 1e-5
        way = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float64)
        quotient = (loss(x + h * way, wi, d) - loss(x - h * way, wi, d)) / (2 * h)
        assert abs(float((dx.double() * way).sum()) - quotient) <= 1e-5 * float((dx.double() * way).abs().sum())
        way = torch.randn(wi.shape, generator=g, device="cuda", dtype=torch.float64)
        quotient = (loss(x, wi + h * way, d) - loss(x, wi - h * way, d)) / (2 * h)
        assert abs(float((dw.double() * way).sum()) - quotient) <= 1e-5 * float((dw.double() * way).abs().sum()) + 1e-5


def test_another_stream(sg):
    q, k, gq, gk, w, pos = made(9, 3000, 8, 2, 128, torch.bfloat16)
    a = (w[0], w[1], *table(500, 128), pos)
    want = sg.sync_qk_norm_rope(q, k, *a) + sg.sync_qk_norm_rope_backward(q, k, gq, gk, *a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = sg.sync_qk_norm_rope(q, k, *a, stream=side) + sg.sync_qk_norm_rope_backward(q, k, gq, gk, *a, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))


def test_no_tokens(sg):
    q, k, gq, gk, w, pos = made(10, 0, 8, 2, 128, torch.bfloat16)
    a = (w[0], w[1], *table(500, 128), pos)
    assert sg.sync_qk_norm_rope(q, k, *a)[0].shape == (0, 8, 128)
    got = sg.sync_qk_norm_rope_backward(q, k, gq, gk, *a)
    assert int(torch.count_nonzero(got[2])) == 0 and int(torch.count_nonzero(got[3])) == 0


def test_refusals(sg):
    q, k, gq, gk, w, pos = made(11, 20, 4, 2, 64, torch.bfloat16)
    cos, sin = table(500, 64)

    def refused(*a, **kw):
        before = sg.kernel_launches()
        with pytest.raises(sg.SyncError) as e:
            sg.sync_qk_norm_rope(*a, **kw)
        assert e.value.status == sg.ERR_ARG and sg.kernel_launches() == before
    refused(q, k[:19], w[0], w[1], cos, sin, pos)
    refused(q, k[..., :32], w[0], w[1], cos, sin, pos)
    refused(q, k.float(), w[0], w[1], cos, sin, pos)
    refused(q[0], k, w[0], w[1], cos, sin, pos)
    refused(q.cpu(), k.cpu(), w[0], w[1], cos, sin, pos)
    refused(q, k, w[0].float(), w[1], cos, sin, pos)
    refused(q, k, w[0][:32], w[1], cos, sin, pos)
    refused(q, k, w[0], w[1], cos, sin[:, :16], pos)
    refused(q, k, w[0], w[1], cos.double(), sin.double(), pos)
    refused(q, k, w[0], w[1], *table(500, 66), pos)          # more than the head
    refused(q, k, w[0], w[1], cos, sin, pos.long())
    refused(q, k, w[0], w[1], cos, sin, pos[:19])
    refused(q, k, w[0], w[1], cos, sin, pos, eps=0.0)
    refused(q, k, w[0], w[1], cos, sin, pos, eps=math.nan)
    refused(q[..., :63], k[..., :63], None, None, *table(500, 62), pos)   # an odd head
    refused(q, k, w[0], w[1], cos, sin, pos, out=(q[:, :3], k))
    wide = torch.zeros(20, 4, 258, device="cuda", dtype=torch.bfloat16)
    refused(wide, wide, None, None, cos, sin, pos)
    with pytest.raises(sg.SyncError):
        sg.sync_qk_norm_rope_backward(q, k, gq[:, :3], gk, w[0], w[1], cos, sin, pos)
