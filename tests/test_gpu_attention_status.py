"""A kernel that gives up waiting: its plan says so.  The waits run out here on
a barrier that nothing arrives on, after a short limit."""
import ctypes

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


def in_vain(sg, plan, tries=3):
    f = sg.lib().syncgb_attn_wait_in_vain
    f.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
    return f(plan.handle, tries, torch.cuda.current_stream().cuda_stream)


def test_a_plan_says_that_a_kernel_gave_up(sg):
    lens, dtype = [5, 130], torch.bfloat16
    q, k, v = (torch.ones(135, h, 64, device="cuda", dtype=dtype) for h in (4, 2, 2))
    plan, other = (sg.sync_attn_plan(lens, lens, 4, 2, 64, dtype, train=True) for _ in range(2))
    o, lse = sg.sync_attn_forward(plan, q, k, v, lse=True)
    sg.sync_attn_backward(plan, q, k, v, o, lse, q)
    torch.cuda.synchronize()
    plan.check()
    assert in_vain(sg, plan) == sg.OK             # the launch is accepted: nothing is known yet
    torch.cuda.synchronize()                      # both of its waits end, the second for want of the first
    before = sg.kernel_launches()
    for call in (plan.check, lambda: sg.sync_attn_forward(plan, q, k, v), lambda: sg.sync_attn_backward(plan, q, k, v, o, lse, q)):
        with pytest.raises(sg.SyncError) as e:
            call()
        assert e.value.status == sg.ERR_CUDA and "gave up" in str(e.value)
    assert sg.kernel_launches() == before
    other.check()                                 # the word is the plan's own, and the device goes on
    assert torch.equal(sg.sync_attn_forward(other, q, k, v), o)
    torch.cuda.synchronize()
    other.check()
    plan.close()
    other.close()


def test_a_replayed_graph_is_asked_the_same_way(sg):
    plan = sg.sync_attn_plan([1], [1], 1, 1, 64, torch.bfloat16)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        assert in_vain(sg, plan) == sg.OK
    torch.cuda.synchronize()
    plan.check()
    graph.replay()
    torch.cuda.synchronize()
    with pytest.raises(sg.SyncError):
        plan.check()
    del graph
    plan.close()
    with pytest.raises(ValueError):
        plan.check()
