"""Plans that are dropped without close(): a finaliser may run anywhere, so it
neither waits for the device nor disturbs a capture."""
import gc

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


def plan_of(sg, lens, heads=4, kv=2, dim=64):
    return sg.sync_attn_plan(lens, lens, heads, kv, dim, torch.bfloat16)


def test_a_plan_dropped_during_a_capture(sg):
    q, k, v = (torch.randn(300, h, 64, device="cuda").bfloat16() for h in (4, 2, 2))
    plan, dropped, out = plan_of(sg, [300]), plan_of(sg, [100, 200]), torch.empty_like(q)
    want = sg.sync_attn_forward(plan, q, k, v)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sg.sync_attn_forward(plan, q, k, v, out=out)
        del dropped
        gc.collect()
        sg.sync_attn_forward(plan, q, k, v, out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    plan.close()


def test_dropping_a_plan_does_not_wait(sg):
    dropped = plan_of(sg, [64])
    torch.cuda.synchronize()
    torch.cuda._sleep(400_000_000)          # about 0.2 s
    del dropped
    gc.collect()
    busy = not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    assert busy


def test_dropped_plans_are_freed_by_the_next_one(sg):
    lens = [4096] * 8                       # a gradient plan of 8 * 4096 rows of 64 heads: 8 MB of row sums
    make = lambda: sg.sync_attn_plan(lens, lens, 64, 64, 64, torch.bfloat16, train=True)  # noqa: E731
    assert make().sizes.device_bytes > 8 << 20
    plan = make()
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    for _ in range(40):                     # 320 MB if they stayed
        plan = make()
    assert torch.cuda.mem_get_info()[0] > free - (64 << 20)
    plan.close()


@pytest.mark.parametrize("device", [None, 0, "cuda", "cuda:0", torch.device("cuda"), torch.device("cuda", 0)], ids=str)
def test_names_of_a_device(sg, device):
    plan = sg.sync_attn_plan([3], [3], 4, 2, 64, torch.bfloat16, device=device)
    assert plan.device == torch.device("cuda", 0)
    x = torch.ones(3, 4, 64, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(sg.sync_attn_forward(plan, x, x[:, :2], x[:, :2]), x)
    plan.close()


def test_a_plan_at_the_interpreter_s_end(sg):
    """A plan that is still there when the program ends leaves quietly."""
    import os
    import subprocess
    import sys
    code = ("import torch, paper_2608_13757_gb300 as sg\n"
            "class Holder: pass\n"
            "h = Holder(); h.me = h\n"
            "h.plan = sg.sync_attn_plan([3], [3], 4, 2, 64, torch.bfloat16)\n"
            "sys = __import__('sys'); sys.keep = sg.sync_attn_plan([3], [3], 4, 2, 64, torch.bfloat16)\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "ignored" not in r.stderr, r.stderr
