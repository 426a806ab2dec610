"""Attention over packed sequences in float16 where most weights are far below the
largest: what thousands of them add together behind a first key that takes the row
has to survive.  Weights are rounded once (2^-11); one too small for float16's
normal numbers is off by half a step of 2^-24 where the largest stands for 2^7 at
least, 2^-32 of it; the result is rounded once.  The norm of a head's errors is that
of independent roundings, uniform within these bounds, half as much again, with
2^-15 of the result for 32-bit arithmetic."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


@pytest.mark.parametrize("causal,train", [(True, False), (True, True), (False, True)], ids=["causal", "causal train", "cross"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("nats", [12.0, 17.0])
def test_small_weights(sg, nats, dtype, causal, train):
    for lq, n, heads, kv, dim in ((200, 8192, 4, 2, 128), (30, 5001, 8, 2, 64), (1000, 3000, 2, 2, 64)):
        g = torch.Generator(device="cuda").manual_seed(51)
        s = 1.0 - 2.0 * (torch.arange(dim, device="cuda") * 7 % 11 % 2)
        k = 0.3 * torch.randn((n, kv, dim), generator=g, device="cuda")
        k[0] = nats / math.sqrt(dim) * s
        v = (0.5 + torch.rand((n, kv, dim), generator=g, device="cuda")) * s
        v[0] *= 1e-3
        q = s + 0.05 * torch.randn((lq, heads, dim), generator=g, device="cuda")
        q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
        plan = sg.sync_attn_plan([lq], [n], heads, kv, dim, dtype, train=train, causal=causal)
        o, lse = sg.sync_attn_forward(plan, q, k, v, lse=True)
        e = torch.einsum("qhd,nhd->hqn", q.double(), k.double().repeat_interleave(heads // kv, 1)) * dim ** -0.5
        if causal:
            e = e.masked_fill(torch.arange(n, device="cuda") > n - lq + torch.arange(lq, device="cuda")[:, None], -math.inf)
        w, vv = torch.softmax(e, -1), v.double().repeat_interleave(heads // kv, 1).transpose(0, 1)
        want, u = w @ vv, torch.finfo(dtype).eps / 2
        tiny = 0.0 if dtype is torch.bfloat16 else 2.0 ** -32
        var = (u * u * (w * w) @ (vv * vv) + (w.amax(-1, keepdim=True) * tiny).square() * vv.square().sum(1, keepdim=True) + (u * want).square()) / 3
        if dtype is torch.float16:
            var = var + 2.0 ** -50
        off = (o.double().transpose(0, 1) - want).square().sum((1, 2)).sqrt()
        allowed = 1.5 * var.sum((1, 2)).sqrt() + 2.0 ** -15 * want.square().sum((1, 2)).sqrt()
        norm = want.square().sum((1, 2)).sqrt()
        assert bool((off <= allowed).all()), f"errors {(off / norm).tolist()} of the heads' norms where {(allowed / norm).tolist()} are allowed"
        # scores: sums of dim products, each addition off by 2^-23 of the sum of sizes (the first key's is the largest)
        exact = torch.logsumexp(e, -1)
        size = (q.double().abs().amax() * k.double().abs().amax() * math.sqrt(dim)).item()
        assert bool(((lse.double() - exact).abs() < 2.0 ** -18 + dim * 2.0 ** -23 * size + 2.0 ** -19 * (1 + exact.abs())).all())
        plan.check()
        plan.close()
