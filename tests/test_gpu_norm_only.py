"""Head norms with nothing to rotate: no table, no position is looked at.

The bound is test_gpu_norm_rope.py's: 32-bit arithmetic, one rounding to the type."""
import ctypes

import pytest
import torch

from tests import attn_reference as ref

pytestmark = pytest.mark.gpu
U = {**ref.U, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def sg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


def made(dtype, dim, n=21, heads=5, kv=2):
    g = torch.Generator(device="cuda").manual_seed(dim)

    def normal(*s):
        return (torch.randn(s, generator=g, device="cuda") * 1.3).to(dtype)
    return normal(n, heads, dim), normal(n, kv, dim), normal(n, heads, dim), normal(n, kv, dim), normal(dim), normal(dim)


def near(got, want, dtype, scale):
    assert bool(((got.double() - want).abs() <= U[dtype] * want.abs() + 2.0 ** -18 * scale + ref.TINY.get(dtype, 0.0)).all())


@pytest.mark.parametrize("rows", [0, 3], ids=["no table", "a shorter table"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
@pytest.mark.parametrize("dim", [128, 34, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
def test_without_a_rotation(sg, dtype, dim, interleaved, rows):
    q, k, gq, gk, wq, wk = made(dtype, dim)
    none = torch.empty(rows, 0, device="cuda")
    for positions in (None, torch.full((q.shape[0],), 1 << 30, dtype=torch.int32, device="cuda")):
        args = (wq, wk, none, none, positions)
        out = sg.sync_qk_norm_rope(q, k, *args, interleaved=interleaved)
        got = sg.sync_qk_norm_rope_backward(q, k, gq, gk, *args, interleaved=interleaved)
        for x, w, y, d, dx, dw in ((q, wq, out[0], gq, got[0], got[2]), (k, wk, out[1], gk, got[1], got[3])):
            x, d, w = x.double(), d.double(), w.double()
            r = (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
            near(y, x * r * w, dtype, (x * r * w).abs().amax(-1, keepdim=True))
            want = r * (d * w - x * r * (d * w * x * r).mean(-1, keepdim=True))
            near(dx, want, dtype, 8 * r * d.abs().amax(-1, keepdim=True) * w.abs().max())
            sizes = (d * x * r).abs().sum((0, 1))
            near(dw, (d * x * r).sum((0, 1)), dtype, sizes)


def test_null_tables(sg):
    """The same through the C call, with every pointer of the table NULL."""
    A, dim, dtype = sg.attention, 64, torch.bfloat16
    q, k, _, _, wq, wk = made(dtype, dim)
    out = torch.full_like(q, 7.0), torch.full_like(k, 7.0)

    def rows(t):
        return A.Rows(t.data_ptr(), t.shape[0], t.stride(0), t.stride(1))
    p = A.NormRope(A.BF16, q.shape[1], k.shape[1], dim, 0, 0, 1e-6, rows(q), rows(k), wq.data_ptr(), wk.data_ptr(), None, None, 0, None)
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert sg.lib().sync_qk_norm_rope(p, rows(out[0]), rows(out[1]), stream) == sg.OK
    for x, w, y in ((q, wq, out[0]), (k, wk, out[1])):
        x = x.double()
        want = x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w.double()
        near(y, want, dtype, want.abs().amax(-1, keepdim=True))
