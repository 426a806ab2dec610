"""Attention calls whose tiles meet nothing, or whose neighbours in the stream
use the same memory."""
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


def normal(seed, *shape, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("q_lens,k_lens", [([0, 0], [5, 131]), ([5, 131], [0, 0]), ([0], [400])], ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
def test_keys_without_queries_and_queries_without_keys(sg, q_lens, k_lens, dtype):
    heads, kv, dim = 4, 2, 64
    q, do = (normal(i, sum(q_lens), heads, dim, dtype=dtype) for i in (1, 2))
    k, v = (normal(i, sum(k_lens), kv, dim, dtype=dtype) for i in (3, 4))
    plan = sg.sync_attn_plan(q_lens, k_lens, heads, kv, dim, dtype, train=True)
    o, lse = sg.sync_attn_forward(plan, q, k, v, lse=True)
    out = tuple(torch.full_like(x, 7.0) for x in (q, k, v))
    sg.sync_attn_backward(plan, q, k, v, o, lse, do, out=out)
    for x in (o,) + out:
        assert int(torch.count_nonzero(x)) == 0
    assert bool((lse == -float("inf")).all())
    plan.close()


def test_gradients_wait_for_the_call_before(sg):
    """The gradients of keys that no query meets are zeros.  Here they go to the
    memory whose contents the call before in the stream reads: it has to have
    read them by then.  (That call leaves SMs free, and both are in the queue
    when it starts, so nothing but the stream's order keeps them apart.)"""
    heads, dim, n, m = 100, 128, 128, 768
    q, k, v = normal(5, n, heads, dim), normal(6, m, heads, dim), normal(7, m, heads, dim)
    plan = sg.sync_attn_plan([n], [m], heads, heads, dim, torch.bfloat16)
    assert plan.sizes.n_splits == 0                    # one kernel, which lets the next one start early
    want = sg.sync_attn_forward(plan, q, k, v)
    keys = sg.sync_attn_plan([0], [m], heads, heads, dim, torch.bfloat16, train=True)
    none, lse = q[:0], torch.empty(heads, 0, device="cuda")
    for _ in range(5):
        a, b, o = k.clone(), v.clone(), torch.empty_like(q)
        torch.cuda.synchronize()
        torch.cuda._sleep(2_000_000)                   # about a millisecond: the calls below are queued meanwhile
        sg.sync_attn_forward(plan, q, a, b, out=o)
        sg.sync_attn_backward(keys, none, k, v, none, lse, none, out=(none, a, b))
        torch.cuda.synchronize()
        assert torch.equal(o, want)
        assert int(torch.count_nonzero(a)) == 0 and int(torch.count_nonzero(b)) == 0
    plan.close()
    keys.close()


def test_lse_off_its_type(sg):
    """Through the C calls: a misaligned lse is refused before any launch."""
    A = sg.attention
    q, k, v = normal(1, 5, 4, 64), normal(2, 5, 2, 64), normal(3, 5, 2, 64)
    plan = sg.sync_attn_plan([5], [5], 4, 2, 64, torch.bfloat16, train=True)
    room = torch.empty(64, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream

    def rows(t):
        return A.Rows(t.data_ptr(), t.shape[0], t.stride(0), t.stride(1))
    before = sg.kernel_launches()
    bad = room.data_ptr() + 2
    assert sg.lib().sync_attn_forward(plan.handle, rows(q), rows(k), rows(v), 0.1, rows(q.clone()), bad, stream) == sg.ERR_ARG
    assert sg.lib().sync_attn_backward(plan.handle, rows(q), rows(k), rows(v), rows(q), bad, rows(q), 0.1, rows(q.clone()), rows(k.clone()), rows(v.clone()), stream) == sg.ERR_ARG
    assert "lse" in sg.lib().sync_last_error().decode() and sg.kernel_launches() == before
    plan.close()
