"""Attention over packed sequences on the GPU against its definition in 64 bits
(attn_reference.py, which derives the bounds), at the lengths, head layouts,
types, strides and masks where tiles and pieces end; its isolation from rows
of other sequences; determinism; and its refusals."""
import math

import pytest
import torch

from tests import attn_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


def starts(lens):
    return [sum(lens[:i]) for i in range(len(lens))]


def inputs(seed, q_rows, k_rows, heads, kv, dim, dtype, gain=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(n, h, std):
        return (torch.randn((n, h, dim), generator=g, device="cuda") * std).to(dtype)
    return normal(q_rows, heads, gain), normal(k_rows, kv, 1.0), normal(k_rows, kv, 1.0), normal(q_rows, heads, 1.0)


def run_and_check(sg, q_lens, k_lens, heads, kv, dim, dtype, train, seed=1, scale=None, gain=1.5):
    q, k, v, do = inputs(seed, sum(q_lens), sum(k_lens), heads, kv, dim, dtype, gain)
    plan = sg.sync_attn_plan(q_lens, k_lens, heads, kv, dim, dtype, train=train)
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
            assert torch.equal(x, y)          # nothing is added in another order
    plan.close()


LENGTHS = {
    "one": ([1], [1]),
    "tile": ([128], [128]),
    "past a tile": ([129, 127, 255, 1], [129, 127, 255, 1]),
    "two tiles and more": ([257, 300, 513], [257, 300, 513]),
    "after earlier keys": ([5, 130, 1, 64], [300, 131, 700, 1000]),
    "fewer keys than queries": ([7, 200, 130], [3, 60, 129]),
    "empty ones": ([0, 5, 4, 0, 9], [5, 0, 4, 0, 131]),
    "single tokens": ([1] * 9, [1, 2, 127, 128, 129, 255, 256, 257, 1111]),
    "a few tokens": ([2, 3, 33, 31], [640, 3, 65, 200]),
}
HEADS = [(1, 1), (4, 4), (8, 2), (6, 2), (5, 1), (16, 1)]


@pytest.mark.parametrize("train", [False, True], ids=["forward", "train"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("lengths", LENGTHS)
def test_lengths(sg, lengths, dim, dtype, train):
    q_lens, k_lens = LENGTHS[lengths]
    run_and_check(sg, q_lens, k_lens, 4, 2, dim, dtype, train)


@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_head_layouts(sg, heads):
    run_and_check(sg, [150, 3, 260], [150, 200, 260], *heads, 128, torch.bfloat16, True)
    run_and_check(sg, [1, 1, 1], [600, 129, 4], *heads, 64, torch.float16, False)


@pytest.mark.parametrize("dim", [8, 16, 24, 40, 56, 72, 80, 96, 104, 120])
def test_head_sizes(sg, dim):
    run_and_check(sg, [140, 20], [140, 300], 4, 2, dim, torch.bfloat16, True)
    run_and_check(sg, [1, 130], [77, 130], 4, 2, dim, torch.float16, True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("q_lens,k_lens", [([1], [9001]), ([1, 1, 1, 1], [40, 5000, 1, 8192]), ([17], [4100]), ([2500], [2500])], ids=str)
def test_long_axes(sg, q_lens, k_lens, dtype):
    run_and_check(sg, q_lens, k_lens, 8, 2, 128, dtype, False)
    run_and_check(sg, q_lens, k_lens, 4, 1, 64, dtype, True)


@pytest.mark.parametrize("gain", [0.0, 12.0, 60.0])
def test_flat_and_peaked_rows(sg, gain):
    """All scores equal, and rows in which one key takes all the weight."""
    run_and_check(sg, [300, 1], [300, 900], 4, 2, 128, torch.bfloat16, True, gain=gain)


def test_scores_that_rise_and_fall(sg):
    """Scores that grow along the keys make every tile raise the running
    maximum by far more than any tolerance of it; falling ones none."""
    n, d = 700, 64
    for sign in (1.0, -1.0):
        q = torch.zeros(n, 2, d, device="cuda", dtype=torch.bfloat16)
        q[..., 0] = sign
        k = torch.zeros(n, 2, d, device="cuda", dtype=torch.bfloat16)
        k[..., 0] = torch.arange(n, device="cuda", dtype=torch.float32)[:, None].to(torch.bfloat16) * 0.5
        v = torch.randn(n, 2, d, device="cuda").to(torch.bfloat16)
        plan = sg.sync_attn_plan([n], [n], 2, 2, d, torch.bfloat16)
        want = ref.packed(q, k, v, [n], [n], [0], [0], 1.0)
        o, lse = sg.sync_attn_forward(plan, q, k, v, scale=1.0, lse=True)
        ref.check(o, want["o"], want["o_tol"], "o")
        ref.check(lse, want["lse"], want["lse_tol"], "lse")


def test_other_scales(sg):
    run_and_check(sg, [200], [333], 4, 2, 128, torch.bfloat16, True, scale=0.3)
    run_and_check(sg, [200], [333], 4, 2, 128, torch.float16, True, scale=1e-3)


@pytest.mark.parametrize("dim", [128, 80])
def test_strided_tensors_and_gaps(sg, dim):
    """Views of a fused projection, sequences in another order with rows between
    them, head-major outputs: rows of no sequence keep what they held."""
    heads, kv, dtype = 8, 2, torch.bfloat16
    q_lens, k_lens, q_starts, k_starts, rows = [130, 1, 77], [130, 300, 90], [200, 7, 60], [400, 5, 310], 640
    g = torch.Generator(device="cuda").manual_seed(3)
    fused = torch.randn((rows, heads + 2 * kv, dim), generator=g, device="cuda").to(dtype)
    q, k, v = fused[:, :heads], fused[:, heads:heads + kv], fused[:, heads + kv:]
    do = torch.randn((heads, rows, dim), generator=g, device="cuda").to(dtype).transpose(0, 1)
    plan = sg.sync_attn_plan(q_lens, k_lens, heads, kv, dim, dtype, q_starts=q_starts, k_starts=k_starts, train=True)
    want = ref.packed(q, k, v, q_lens, k_lens, q_starts, k_starts, dim ** -0.5, do)
    out = torch.full((heads, rows, dim), 7.0, dtype=dtype, device="cuda").transpose(0, 1)
    lse = torch.full((heads, rows), 7.0, device="cuda")
    sg.sync_attn_forward(plan, q, k, v, out=out, lse=lse)
    grads = (torch.full_like(out, 7.0), torch.full((rows, kv, dim), 7.0, dtype=dtype, device="cuda"), torch.full((rows, 3, dim), 7.0, dtype=dtype, device="cuda")[:, 1:])
    sg.sync_attn_backward(plan, q, k, v, out, lse, do, out=grads)
    for x, name in zip((out, lse) + grads, ("o", "lse", "dq", "dk", "dv")):
        ref.check(x, want[name], want[name + "_tol"], name)
        assert bool((x[torch.isnan(want[name])] == 7.0).all()), name
    o2, lse2 = sg.sync_attn_forward(plan, q, k, v, lse=True)     # allocated by the call: zero between the sequences
    assert bool((o2[torch.isnan(want["o"])] == 0).all()) and bool((lse2[torch.isnan(want["lse"])] == -math.inf).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf, torch.finfo(torch.bfloat16).min])
def test_other_rows_do_not_reach_a_sequence(sg, bad):
    """Rows before, between and after the sequences hold NaN, infinities or the
    type's lowest value, and so does one whole sequence: the others' outputs
    and gradients are those of a clean tensor, bit for bit."""
    heads, kv, dim, dtype = 4, 2, 128, torch.bfloat16
    q_lens, k_lens, q_starts, k_starts = [100, 60, 131, 1], [100, 260, 131, 70], [3, 110, 170, 310], [1, 110, 380, 520]
    tensors = inputs(5, 330, 600, heads, kv, dim, dtype)
    results = []
    for dirty in (False, True):
        q, k, v, do = (t.clone() for t in tensors)
        for t, at, lens in ((q, q_starts, q_lens), (do, q_starts, q_lens), (k, k_starts, k_lens), (v, k_starts, k_lens)):
            mine = torch.zeros(t.shape[0], dtype=torch.bool, device="cuda")
            for i in (0, 2, 3):
                mine[at[i]:at[i] + lens[i]] = True
            t[~mine] = bad if dirty else 1.0
        plan = sg.sync_attn_plan(q_lens, k_lens, heads, kv, dim, dtype, q_starts=q_starts, k_starts=k_starts, train=True)
        o, lse = sg.sync_attn_forward(plan, q, k, v, lse=True)
        results.append((o, lse.t()) + sg.sync_attn_backward(plan, q, k, v, o, lse, do))
        infer = sg.sync_attn_plan(q_lens, k_lens, heads, kv, dim, dtype, q_starts=q_starts, k_starts=k_starts)
        assert torch.equal(sg.sync_attn_forward(infer, q, k, v)[3:103], o[3:103])
    for x, y, at, lens in zip(*results, (q_starts, q_starts, q_starts, k_starts, k_starts), (q_lens, q_lens, q_lens, k_lens, k_lens)):
        for i in (0, 2, 3):
            a, b = x[at[i]:at[i] + lens[i]], y[at[i]:at[i] + lens[i]]
            assert bool(torch.isfinite(a).all()) and torch.equal(a, b)


def test_keys_that_are_hidden_do_not_reach_a_row(sg):
    """A NaN or infinite key reaches the queries that see it, and no other."""
    n, at = 300, 200
    q, k, v, _ = inputs(7, n, n, 2, 1, 64, torch.float16)
    plan = sg.sync_attn_plan([n], [n], 2, 1, 64, torch.float16)
    clean = sg.sync_attn_forward(plan, q, k, v)
    k[at] = math.nan
    o = sg.sync_attn_forward(plan, q, k, v)
    assert torch.equal(o[:at], clean[:at]) and bool(torch.isnan(o[at:]).all())


def test_shared_keys(sg):
    """Sequences that read the same key rows."""
    heads, kv, dim, dtype = 8, 2, 128, torch.bfloat16
    q, k, v, _ = inputs(8, 3, 500, heads, kv, dim, dtype)
    args = ([1, 1, 1], [400, 500, 256], [0, 1, 2], [0, 0, 100])
    plan = sg.sync_attn_plan(args[0], args[1], heads, kv, dim, dtype, q_starts=args[2], k_starts=args[3])
    want = ref.packed(q, k, v, *args, dim ** -0.5)
    ref.check(sg.sync_attn_forward(plan, q, k, v), want["o"], want["o_tol"], "o")
    with pytest.raises(sg.SyncError) as e:
        sg.sync_attn_plan(args[0], args[1], heads, kv, dim, dtype, q_starts=args[2], k_starts=args[3], train=True)
    assert e.value.status == sg.ERR_MALFORMED


def test_offsets_past_32_bits(sg):
    """Keys that start past 2^31 entries, 4 GB into the cache."""
    heads, kv, dim, dtype, rows = 4, 8, 128, torch.bfloat16, 2_200_000
    heads = 8
    k = torch.zeros((rows, kv, dim), dtype=dtype, device="cuda")
    v = torch.zeros((rows, kv, dim), dtype=dtype, device="cuda")
    q_lens, k_lens, k_starts = [1, 150], [700, 260], [rows - 1000, rows - 260]
    q, kk, vv, do = inputs(9, 151, 1000, heads, kv, dim, dtype)
    k[-1000:], v[-1000:] = kk, vv
    plan = sg.sync_attn_plan(q_lens, k_lens, heads, kv, dim, dtype, k_starts=k_starts, train=True)
    want = ref.packed(q, kk, vv, q_lens, k_lens, [0, 1], [0, 740], dim ** -0.5, do)
    o, lse = sg.sync_attn_forward(plan, q, k, v, lse=True)
    ref.check(o, want["o"], want["o_tol"], "o")
    dq, dk, dv = sg.sync_attn_backward(plan, q, k, v, o, lse, do)
    ref.check(dq, want["dq"], want["dq_tol"], "dq")
    for x, name in ((dk, "dk"), (dv, "dv")):
        ref.check(x[-1000:], want[name], want[name + "_tol"], name)
        assert int(torch.count_nonzero(x[:-1000])) == 0


def test_gradients_against_differences(sg):
    """The gradients' product with a direction against the difference quotient
    of the 64-bit forward pass along it."""
    q_lens, k_lens, heads, kv, dim, dtype = [70, 130], [70, 200], 4, 2, 64, torch.float16
    q, k, v, do = inputs(11, 200, 270, heads, kv, dim, dtype)
    plan = sg.sync_attn_plan(q_lens, k_lens, heads, kv, dim, dtype, train=True)
    o, lse = sg.sync_attn_forward(plan, q, k, v, lse=True)
    grads = sg.sync_attn_backward(plan, q, k, v, o, lse, do)
    want = ref.packed(q, k, v, q_lens, k_lens, starts(q_lens), starts(k_lens), dim ** -0.5, do)

    def loss(t):
        total = 0.0
        for n, m, a, b in zip(q_lens, k_lens, starts(q_lens), starts(k_lens)):
            for h in range(heads):
                x, y, z = t[0][a:a + n, h], t[1][b:b + m, h // 2], t[2][b:b + m, h // 2]
                s = (x @ y.T * dim ** -0.5).masked_fill(~ref.visible(n, m, x.device), -math.inf)
                total += float((torch.softmax(s, 1) @ z * do[a:a + n, h].double()).sum())
        return total
    base = [x.double() for x in (q, k, v)]
    g = torch.Generator(device="cuda").manual_seed(12)
    for i, name in enumerate(("dq", "dk", "dv")):
        way = torch.randn(base[i].shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-4
        moved = [[x + (s * h * way if j == i else 0) for j, x in enumerate(base)] for s in (1, -1)]
        quotient = (loss(moved[0]) - loss(moved[1])) / (2 * h)
        allowed = float((want[name + "_tol"] * way.abs()).sum()) + 1e-5 * abs(quotient) + 1e-5
        assert abs(float((grads[i].double() * way).sum()) - quotient) <= allowed, name


def test_another_stream(sg):
    q, k, v, do = inputs(13, 900, 900, 8, 2, 128, torch.bfloat16)
    plan = sg.sync_attn_plan([900], [900], 8, 2, 128, torch.bfloat16, train=True)
    o, lse = sg.sync_attn_forward(plan, q, k, v, lse=True)
    want = sg.sync_attn_backward(plan, q, k, v, o, lse, do)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        a, b = sg.sync_attn_forward(plan, q, k, v, lse=True, stream=stream)
        got = sg.sync_attn_backward(plan, q, k, v, a, b, do, stream=stream)
        side.synchronize()
        for x, y in zip((o, lse) + want, (a, b) + got):
            assert torch.equal(x, y)


def test_in_a_graph(sg):
    """Calls are captured: they allocate nothing and wait for nothing."""
    q, k, v, _ = inputs(14, 4, 2000, 8, 2, 128, torch.bfloat16)
    plan = sg.sync_attn_plan([1] * 4, [500] * 4, 8, 2, 128, torch.bfloat16)
    out = torch.empty_like(q)
    want = sg.sync_attn_forward(plan, q, k, v)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sg.sync_attn_forward(plan, q, k, v, out=out)
    for _ in range(3):
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refusals(sg):
    q, k, v, do = inputs(15, 10, 20, 4, 2, 64, torch.bfloat16)
    plan = sg.sync_attn_plan([10], [20], 4, 2, 64, torch.bfloat16)

    def refused(f, status=None):
        before = sg.kernel_launches()
        with pytest.raises(sg.SyncError) as e:
            f()
        assert e.value.status == (sg.ERR_ARG if status is None else status) and sg.kernel_launches() == before
        return str(e.value)
    f = sg.sync_attn_forward
    refused(lambda: f(plan, q[:9], k, v))                       # fewer rows than the plan needs
    refused(lambda: f(plan, q, k[:19], v))
    refused(lambda: f(plan, q.float(), k, v))
    refused(lambda: f(plan, q, k.to(torch.float16), v))
    refused(lambda: f(plan, q[:, :3], k, v))                    # heads
    refused(lambda: f(plan, q[..., :32], k, v))
    refused(lambda: f(plan, q.cpu(), k, v))
    refused(lambda: f(plan, q, k, v, scale=0.0))
    refused(lambda: f(plan, q, k, v, scale=math.nan))
    refused(lambda: f(plan, q, k, v, out=torch.empty(10, 4, 64, device="cuda")))
    refused(lambda: f(plan, q, k, v, lse=torch.empty(4, 9, device="cuda")))
    wide = torch.zeros(10, 4, 72, device="cuda", dtype=torch.bfloat16)
    refused(lambda: f(plan, wide[..., 4:68], k, v))             # 8 bytes off a 16-byte boundary
    odd = torch.zeros(10, 4 * 64 + 4, device="cuda", dtype=torch.bfloat16)[:, :256].view(10, 4, 64)
    refused(lambda: f(plan, odd, k, v))                         # rows 8 bytes off
    refused(lambda: f(plan, torch.zeros(10, 64, 4, device="cuda", dtype=torch.bfloat16).transpose(1, 2), k, v))
    o, lse = f(plan, q, k, v, lse=True)
    assert "train" in refused(lambda: sg.sync_attn_backward(plan, q, k, v, o, lse, do))
    p = sg.sync_attn_plan
    bf = torch.bfloat16
    refused(lambda: p([1], [1, 2], 4, 2, 64, bf))
    refused(lambda: p([-1], [1], 4, 2, 64, bf))
    refused(lambda: p([1], [1], 4, 3, 64, bf))
    refused(lambda: p([1], [1], 0, 0, 64, bf))
    refused(lambda: p([1], [1], 4, 2, 136, bf))
    refused(lambda: p([1], [1], 4, 2, 60, bf))
    refused(lambda: p([1], [1], 4, 2, 64, torch.float32))
    refused(lambda: p([1], [1], 4, 2, 64, torch.int32))
    refused(lambda: p([1], [1], 4, 2, 64, bf, q_starts=[-1]))
    refused(lambda: p([4, 4], [4, 4], 4, 2, 64, bf, q_starts=[0, 3]), sg.ERR_MALFORMED)
    refused(lambda: p([4], [4], 4, 2, 64, bf, k_starts=[(1 << 31) - 3]), sg.ERR_OVERFLOW)
    plan.close()
    with pytest.raises(ValueError):
        f(plan, q, k, v)


def test_nothing_to_do(sg):
    plan = sg.sync_attn_plan([], [], 4, 2, 64, torch.bfloat16, train=True)
    e = torch.empty(0, 4, 64, device="cuda", dtype=torch.bfloat16)
    z = torch.empty(0, 2, 64, device="cuda", dtype=torch.bfloat16)
    o, lse = sg.sync_attn_forward(plan, e, z, z, lse=True)
    assert o.shape == (0, 4, 64)
    assert [x.shape[0] for x in sg.sync_attn_backward(plan, e, z, z, o, lse, e)] == [0, 0, 0]
