"""Attention to another sequence's states on the GPU (every query sees all keys
of its sequence) against its definition in 64 bits, at lengths where tiles and
pieces end, with its gradients, shared states, and rows of other sequences.
The bounds are attn_reference's; only its mask is replaced."""
import math

import pytest
import torch

from tests import attn_reference as ref
from tests import gradient_norms as norms

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


@pytest.fixture(autouse=True)
def all_seen(monkeypatch):
    monkeypatch.setattr(ref, "visible", lambda n, m, device: torch.ones(n, m, dtype=torch.bool, device=device))


def starts(lens):
    return [sum(lens[:i]) for i in range(len(lens))]


def inputs(seed, q_rows, k_rows, heads, kv, dim, dtype, gain=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(n, h, std=1.0):
        return (torch.randn((n, h, dim), generator=g, device="cuda") * std).to(dtype)
    return normal(q_rows, heads, gain), normal(k_rows, kv), normal(k_rows, kv), normal(q_rows, heads)


def run_and_check(sg, q_lens, k_lens, heads, kv, dim, dtype, train=True, seed=1, scale=None, gain=1.5):
    q, k, v, do = inputs(seed, sum(q_lens), sum(k_lens), heads, kv, dim, dtype, gain)
    plan = sg.sync_attn_plan(q_lens, k_lens, heads, kv, dim, dtype, train=train, causal=False)
    assert plan.sizes.pairs == sum(x * y for x, y in zip(q_lens, k_lens))
    want = ref.packed(q, k, v, q_lens, k_lens, starts(q_lens), starts(k_lens), scale or dim ** -0.5, do if train else None)
    o, lse = sg.sync_attn_forward(plan, q, k, v, scale=scale, lse=True)
    ref.check(o, want["o"], want["o_tol"], "o")
    ref.check(lse, want["lse"], want["lse_tol"], "lse")
    assert torch.equal(sg.sync_attn_forward(plan, q, k, v, scale=scale), o)
    if train:
        grads = sg.sync_attn_backward(plan, q, k, v, o, lse, do, scale=scale)
        for x, name in zip(grads, ("dq", "dk", "dv")):
            ref.check(x, want[name], want[name + "_tol"], name)
        for x, y in zip(sg.sync_attn_backward(plan, q, k, v, o, lse, do, scale=scale), grads):
            assert torch.equal(x, y)
    plan.check()
    plan.close()


LENGTHS = {
    "one": ([1], [1]),
    "tiles": ([128, 256], [256, 128]),
    "more keys": ([129, 127, 1, 300], [700, 128, 257, 301]),
    "more queries": ([700, 300, 257, 130], [1, 127, 129, 128]),
    "second tile past the keys": ([256, 200], [130, 3]),
    "no keys, no queries": ([5, 0, 200, 0], [0, 300, 0, 0]),
    "single tokens": ([1] * 6, [1, 127, 128, 129, 1500, 513]),
    "a few tokens": ([2, 3, 33, 5], [640, 3, 65, 1500]),
}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("lengths", LENGTHS)
def test_lengths(sg, lengths, dim, dtype):
    q_lens, k_lens = LENGTHS[lengths]
    run_and_check(sg, q_lens, k_lens, 4, 2, dim, dtype)
    run_and_check(sg, q_lens, k_lens, 4, 4, dim, dtype, train=False)


@pytest.mark.parametrize("heads", [(1, 1), (4, 4), (8, 2), (6, 2), (5, 1), (16, 1)], ids=str)
def test_head_layouts(sg, heads):
    run_and_check(sg, [150, 3, 260], [90, 300, 260], *heads, 80, torch.bfloat16)
    run_and_check(sg, [1, 1, 1], [600, 129, 4], *heads, 64, torch.float16, train=False)


@pytest.mark.parametrize("q_lens,k_lens", [([1], [9001]), ([1, 1, 1, 1], [40, 5000, 1, 8192]), ([17], [4100]), ([2500], [140]), ([130, 900], [2500, 33])], ids=str)
def test_long_axes(sg, q_lens, k_lens):
    run_and_check(sg, q_lens, k_lens, 8, 2, 128, torch.bfloat16, train=False)
    run_and_check(sg, q_lens, k_lens, 4, 1, 64, torch.float16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
def test_norms_of_the_errors(sg, dtype, monkeypatch):
    """The norm of each head's error, which a factor of 0.95 or a mask that is
    off by one exceeds (gradient_norms takes its mask from attn_reference)."""
    q_lens, k_lens, heads, kv, dim = [129, 40, 300], [257, 500, 33], 4, 2, 64
    q, k, v, do = inputs(3, sum(q_lens), sum(k_lens), heads, kv, dim, dtype)
    plan = sg.sync_attn_plan(q_lens, k_lens, heads, kv, dim, dtype, train=True, causal=False)
    o, lse = sg.sync_attn_forward(plan, q, k, v, lse=True)
    norms.check((o,) + sg.sync_attn_backward(plan, q, k, v, o, lse, do), q, k, v, do, q_lens, k_lens, dim ** -0.5)


def test_shared_states(sg):
    """Several decoders of one encoder's states; a gradient would add to the same rows."""
    heads, kv, dim, dtype = 8, 8, 64, torch.bfloat16
    q, k, v, _ = inputs(8, 9, 500, heads, kv, dim, dtype)
    args = ([1, 1, 7], [400, 400, 500], [0, 1, 2], [0, 0, 0])
    plan = sg.sync_attn_plan(args[0], args[1], heads, kv, dim, dtype, q_starts=args[2], k_starts=args[3], causal=False)
    want = ref.packed(q, k, v, *args, dim ** -0.5)
    ref.check(sg.sync_attn_forward(plan, q, k, v), want["o"], want["o_tol"], "o")
    with pytest.raises(sg.SyncError) as e:
        sg.sync_attn_plan(args[0], args[1], heads, kv, dim, dtype, q_starts=args[2], k_starts=args[3], train=True, causal=False)
    assert e.value.status == sg.ERR_MALFORMED


@pytest.mark.parametrize("bad", [math.nan, math.inf, torch.finfo(torch.bfloat16).min])
def test_other_rows_do_not_reach_a_sequence(sg, bad):
    heads, kv, dim, dtype = 4, 2, 128, torch.bfloat16
    q_lens, k_lens, q_starts, k_starts = [100, 60, 261, 1], [90, 260, 131, 70], [3, 110, 170, 440], [1, 110, 380, 520]
    tensors = inputs(5, 450, 600, heads, kv, dim, dtype)
    results = []
    for dirty in (False, True):
        q, k, v, do = (t.clone() for t in tensors)
        for t, at, lens in ((q, q_starts, q_lens), (do, q_starts, q_lens), (k, k_starts, k_lens), (v, k_starts, k_lens)):
            mine = torch.zeros(t.shape[0], dtype=torch.bool, device="cuda")
            for i in (0, 2, 3):
                mine[at[i]:at[i] + lens[i]] = True
            t[~mine] = bad if dirty else 1.0
        plan = sg.sync_attn_plan(q_lens, k_lens, heads, kv, dim, dtype, q_starts=q_starts, k_starts=k_starts, train=True, causal=False)
        o, lse = sg.sync_attn_forward(plan, q, k, v, lse=True)
        results.append((o, lse.t()) + sg.sync_attn_backward(plan, q, k, v, o, lse, do))
    for x, y, at, lens in zip(*results, (q_starts, q_starts, q_starts, k_starts, k_starts), (q_lens, q_lens, q_lens, k_lens, k_lens)):
        for i in (0, 2, 3):
            a, b = x[at[i]:at[i] + lens[i]], y[at[i]:at[i] + lens[i]]
            assert bool(torch.isfinite(a).all()) and torch.equal(a, b)


def test_graph_and_stream(sg):
    q, k, v, _ = inputs(14, 4, 2000, 8, 8, 64, torch.bfloat16)
    plan = sg.sync_attn_plan([1] * 4, [500] * 4, 8, 8, 64, torch.bfloat16, causal=False)
    out, want = torch.empty_like(q), sg.sync_attn_forward(plan, q, k, v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sg.sync_attn_forward(plan, q, k, v, out=out)
    graph.replay()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = sg.sync_attn_forward(plan, q, k, v, stream=side)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(other, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [8, 40, 64, 80, 128])
@pytest.mark.parametrize("heads,kv", [(4, 4), (16, 1), (6, 2), (20, 10)], ids=str)
def test_few_queries(sg, heads, kv, dim, dtype):
    """Up to 16 rows of a key head go to a kernel of their own."""
    run_and_check(sg, [1, 1, 0, 1, 1], [100, 0, 30, 1, 700], heads, kv, dim, dtype, train=False)
    if heads // kv <= 4:
        run_and_check(sg, [4, 1, 3], [129, 0, 2000], heads, kv, dim, dtype, train=False)


def test_few_queries_in_strided_rows(sg):
    """Values where a projection left them, head-major keys, gaps between and
    NaN behind the sequences: rows of no sequence keep what they held."""
    heads, kv, dim, dtype = 8, 4, 64, torch.bfloat16
    q_lens, k_lens, q_starts, k_starts = [2, 1, 8], [300, 5, 131], [9, 0, 20], [400, 20, 40]
    q, k, v, _ = inputs(21, 30, 701, heads, kv, dim, dtype)
    wide = torch.full((701, 3 * kv, dim), math.nan, dtype=dtype, device="cuda")
    k = k.transpose(0, 1).contiguous().transpose(0, 1)
    for a, n in zip(k_starts, k_lens):
        wide[a:a + n, kv:2 * kv] = v[a:a + n]
    want = ref.packed(q, k, v, q_lens, k_lens, q_starts, k_starts, dim ** -0.5)
    for other in (0.0, math.nan):
        mine = torch.zeros(701, dtype=torch.bool, device="cuda")
        for a, n in zip(k_starts, k_lens):
            mine[a:a + n] = True
        k[~mine] = other
        plan = sg.sync_attn_plan(q_lens, k_lens, heads, kv, dim, dtype, q_starts=q_starts, k_starts=k_starts, causal=False)
        out, lse = torch.full((30, heads + 1, dim), 7.0, dtype=dtype, device="cuda")[:, 1:], torch.full((heads, 30), 7.0, device="cuda")
        sg.sync_attn_forward(plan, q, k, wide[:, kv:2 * kv], out=out, lse=lse)
        ref.check(out, want["o"], want["o_tol"], "o")
        ref.check(lse, want["lse"], want["lse_tol"], "lse")
        none = torch.isnan(want["o"])
        assert bool((out[none] == 7).all()) and bool((lse[torch.isnan(want["lse"])] == 7).all())


def test_few_queries_many_and_long(sg):
    run_and_check(sg, [1] * 300, [(i * 53) % 400 for i in range(300)], 4, 4, 64, torch.float16, train=False)
    run_and_check(sg, [1, 2], [40000, 9], 8, 2, 128, torch.bfloat16, train=False)


def test_few_queries_past_32_bits(sg):
    """Keys and values behind the first 2^31 entries of their tensors."""
    heads, kv, dim, rows, n = 8, 8, 128, (1 << 21) + 500, 400
    q, k, v, _ = inputs(31, 2, n, heads, kv, dim, torch.bfloat16)
    plan = sg.sync_attn_plan([2], [n], heads, kv, dim, torch.bfloat16, causal=False)
    want = sg.sync_attn_forward(plan, q, k, v)
    far = sg.sync_attn_plan([2], [n], heads, kv, dim, torch.bfloat16, k_starts=[rows - n], causal=False)
    large = torch.empty((2, rows, kv, dim), dtype=torch.bfloat16, device="cuda")
    large[0, rows - n:], large[1, rows - n:] = k, v
    assert torch.equal(sg.sync_attn_forward(far, q, large[0], large[1]), want)


def test_few_queries_while_an_encoder_changes(sg):
    """A captured step reads what the states hold when it is replayed."""
    q_lens, k_lens, heads, kv, dim = [1, 2, 0, 1], [700, 20, 9, 0], 8, 4, 64
    q, k, v, _ = inputs(32, 4, 729, heads, kv, dim, torch.float16)
    plan = sg.sync_attn_plan(q_lens, k_lens, heads, kv, dim, torch.float16, causal=False)
    out, lse = torch.empty_like(q), torch.empty((heads, 4), device="cuda")
    sg.sync_attn_forward(plan, q, k, v, out=out, lse=lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sg.sync_attn_forward(plan, q, k, v, out=out, lse=lse)
    for seed in (33, 34):
        for t, new in zip((q, k, v), inputs(seed, 4, 729, heads, kv, dim, torch.float16)):
            t.copy_(new)
        graph.replay()
        want = ref.packed(q, k, v, q_lens, k_lens, starts(q_lens), starts(k_lens), dim ** -0.5)
        ref.check(out, want["o"], want["o_tol"], "o")
        ref.check(lse, want["lse"], want["lse_tol"], "lse")
