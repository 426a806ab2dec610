"""The operators record nothing for autograd, and say so where a gradient would
be lost in silence."""
import warnings

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


@pytest.fixture
def calls(sg):
    """{name: (inputs, the call on them)}"""
    q, k, v = (torch.randn(9, h, 64, device="cuda").bfloat16() for h in (4, 2, 2))
    w = torch.ones(64, device="cuda").bfloat16()
    cos, sin = torch.ones(9, 32, device="cuda"), torch.zeros(9, 32, device="cuda")
    plan = sg.sync_attn_plan([9], [9], 4, 2, 64, torch.bfloat16)
    yield {"sync_attn_forward": ((q, k, v), lambda *x: sg.sync_attn_forward(plan, *x)),
           "sync_qk_norm_rope": ((q, k, w, w.clone()), lambda *x: sg.sync_qk_norm_rope(*x, cos, sin)[0])}
    plan.close()


@pytest.mark.parametrize("name", ["sync_attn_forward", "sync_qk_norm_rope"])
def test_lost_gradients_are_said(calls, name):
    inputs, call = calls[name]
    want = call(*inputs)
    for i in range(len(inputs)):
        x = [t.clone().requires_grad_() if i == j else t for j, t in enumerate(inputs)]
        with pytest.warns(UserWarning, match=f"{name} records nothing"):
            y = call(*x)
        assert torch.equal(y, want) and not y.requires_grad


@pytest.mark.parametrize("name", ["sync_attn_forward", "sync_qk_norm_rope"])
def test_no_word_where_none_is_lost(calls, name):
    inputs, call = calls[name]
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        call(*inputs)
        with torch.no_grad():
            call(*(t.clone().requires_grad_() for t in inputs))
        call(*(t.clone().requires_grad_().detach() for t in inputs))


def test_in_a_function_of_its_own(sg):
    """The usual way to record them: forward and backward calls in a Function."""
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
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        o = Attention.apply(q, k, v)
        o.backward(do)
    with torch.no_grad():
        o, lse = sg.sync_attn_forward(plan, q, k, v, lse=True)
        for x, y in zip((q, k, v), sg.sync_attn_backward(plan, q, k, v, o, lse, do)):
            assert torch.equal(x.grad, y)
    plan.close()
