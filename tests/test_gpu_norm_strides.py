"""Head norms on views: interleaved pairs off every wide boundary, and inputs
that repeat a row or a head.  Bounds as in test_gpu_norm_rope.py."""
import pytest
import torch

from tests.test_gpu_norm_rope import DTYPES, made, run_and_check, sg, table  # noqa: F401  (sg is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shift", [0, 1, 3, 4, 8])
@pytest.mark.parametrize("dim,rotated", [(128, 128), (96, 96), (80, 40)])
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp16", "fp32"])
def test_interleaved_views(sg, dtype, dim, rotated, shift):  # noqa: F811
    n, heads, kv = 67, 6, 2
    g = torch.Generator(device="cuda").manual_seed(2)
    flat = torch.randn((2, n, (heads + 2 * kv) * dim + 8 + shift), generator=g, device="cuda").to(dtype)
    view = flat[:, :, shift:shift + (heads + 2 * kv) * dim].unflatten(2, (heads + 2 * kv, dim))
    w = [torch.ones(dim, device="cuda", dtype=dtype) * 1.1, torch.ones(dim + 1, device="cuda", dtype=dtype)[1:]]
    pos = torch.arange(n, device="cuda", dtype=torch.int32) * 3
    run_and_check(sg, view[0, :, :heads], view[0, :, heads:heads + kv], view[1, :, :heads], view[1, :, heads:heads + kv], w, *table(500, rotated), pos, True)


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
def test_broadcast_inputs(sg, interleaved):  # noqa: F811
    n, heads, kv, dim = 50, 6, 2, 128
    q, k, gq, gk, w, pos = made(3, n, heads, kv, dim, torch.bfloat16)
    run_and_check(sg, q[:1].expand(n, -1, -1), k[:, :1].expand(-1, kv, -1), gq[:, :1].expand(-1, heads, -1), gk[:1].expand(n, -1, -1), w, *table(500, dim), pos, interleaved)


def test_broadcast_outputs_are_refused(sg):  # noqa: F811
    n, heads, kv, dim = 50, 6, 2, 128
    q, k, gq, gk, w, pos = made(3, n, heads, kv, dim, torch.bfloat16)
    args = (w[0], w[1], *table(500, dim), pos)
    for out in ((q[:1].expand(n, -1, -1), k), (q, k[:, :1].expand(-1, kv, -1))):
        for call in (lambda: sg.sync_qk_norm_rope(q, k, *args, out=out), lambda: sg.sync_qk_norm_rope_backward(q, k, gq, gk, *args, out=out)):  # noqa: B023
            before = sg.kernel_launches()
            with pytest.raises(sg.SyncError) as e:
                call()
            assert e.value.status == sg.ERR_ARG and sg.kernel_launches() == before
