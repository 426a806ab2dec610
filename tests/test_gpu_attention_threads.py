"""The operators' calls from threads that have used no GPU before, as an
autograd backward pass makes them."""
import threading

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


def in_a_thread(f):
    got = []

    def run():
        try:
            got.append(f())
        except Exception as e:
            got.append(e)
    t = threading.Thread(target=run)
    t.start()
    t.join()
    if isinstance(got[0], Exception):
        raise got[0]
    return got[0]


def test_each_call_is_a_thread_s_first(sg):
    lens, heads, kv, dim = [70, 5], 4, 2, 64
    q, k, v, do = (torch.randn(75, h, dim, device="cuda").bfloat16() for h in (heads, kv, kv, heads))
    w = torch.ones(dim, device="cuda").bfloat16()
    table = torch.ones(75, dim // 2, device="cuda"), torch.zeros(75, dim // 2, device="cuda")
    plan = sg.sync_attn_plan(lens, lens, heads, kv, dim, torch.bfloat16, train=True)
    o, lse = sg.sync_attn_forward(plan, q, k, v, lse=True)
    # outputs are given, so that the call is the thread's first use of the GPU
    empty = [torch.empty_like(x) for x in (o, q, k, v)]
    calls = {
        "forward": (lambda out: sg.sync_attn_forward(plan, q, k, v, out=out), o, torch.empty_like(o)),
        "backward": (lambda out: sg.sync_attn_backward(plan, q, k, v, o, lse, do, out=out),
                     sg.sync_attn_backward(plan, q, k, v, o, lse, do), tuple(empty[1:])),
        "norm": (lambda out: sg.sync_qk_norm_rope(q, k, w, w, *table, out=out), sg.sync_qk_norm_rope(q, k, w, w, *table), (empty[0], torch.empty_like(k))),
        "norm gradient": (lambda out: sg.sync_qk_norm_rope_backward(q, k, do, v, w, w, *table, out=out),
                          sg.sync_qk_norm_rope_backward(q, k, do, v, w, w, *table), (torch.empty_like(q), torch.empty_like(k))),
    }
    for name, (call, want, out) in calls.items():
        got = in_a_thread(lambda: call(out))  # noqa: B023
        torch.cuda.synchronize()
        for x, y in zip(got if isinstance(got, tuple) else (got,), want if isinstance(want, tuple) else (want,)):
            assert torch.equal(x, y), name
    other = in_a_thread(lambda: sg.sync_attn_plan(lens, lens, heads, kv, dim, torch.bfloat16, train=True, device=0))
    assert torch.equal(in_a_thread(lambda: sg.sync_attn_forward(other, q, k, v)), o)
    in_a_thread(other.check)
    in_a_thread(other.close)
    plan.close()


def test_a_backward_pass(sg):
    """Forward and backward calls in an autograd Function."""
    lens, heads, kv, dim = [70, 5], 4, 2, 64
    plan = sg.sync_attn_plan(lens, lens, heads, kv, dim, torch.bfloat16, train=True)

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            o, lse = sg.sync_attn_forward(plan, q, k, v, lse=True)
            ctx.save_for_backward(q, k, v, o, lse)
            return o

        @staticmethod
        def backward(ctx, do):
            return sg.sync_attn_backward(plan, *ctx.saved_tensors, do)
    q, k, v = (torch.randn(75, h, dim, device="cuda").bfloat16().requires_grad_() for h in (heads, kv, kv))
    do = torch.randn(75, heads, dim, device="cuda").bfloat16()
    o = Attention.apply(q, k, v)
    o.backward(do)
    with torch.no_grad():
        o, lse = sg.sync_attn_forward(plan, q, k, v, lse=True)
        for x, y in zip((q, k, v), sg.sync_attn_backward(plan, q, k, v, o, lse, do)):
            assert torch.equal(x.grad, y)
    plan.close()
