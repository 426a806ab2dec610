"""The attention block's operators together with the programs of their tile
walk, as examples/packed_attention.py runs them."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle
import workloads
from tests import attn_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13757_gb300 import build
    build.build()
    spec = importlib.util.spec_from_file_location("packed_attention", os.path.join(ROOT, "examples", "packed_attention.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("lengths", [[1], [128, 129], [300, 1, 0, 257]], ids=str)
def test_block(example, lengths):
    """Every step against its definition on the step's own inputs."""
    heads, kv, dim = 8, 2, 128
    r = example.block(lengths, heads, kv, dim)
    starts = [sum(lengths[:i]) for i in range(len(lengths))]
    wq, wk, cos, sin, positions = r["norm"]
    u = ref.U[torch.bfloat16]
    for x, w, y in ((r["q"], wq, r["qn"]), (r["k"], wk, r["kn"])):
        want = ref.norm_rope(x, w, cos, sin, positions, 1e-6, False)
        assert bool(((y.double() - want).abs() <= u * want.abs() + 2.0 ** -18 * want.abs().amax(-1, keepdim=True)).all())
    want = ref.packed(r["qn"], r["kn"], r["v"], lengths, lengths, starts, starts, dim ** -0.5, r["do"])
    for name, got in (("o", r["o"]), ("dq", r["dqn"]), ("dk", r["dkn"]), ("dv", r["dv"])):
        ref.check(got, want[name], want[name + "_tol"], name)
    for name in ("dq", "dk", "dwq", "dwk"):
        assert bool(torch.isfinite(r[name]).all())
    r["plan"].close()


def test_schedule(example):
    """The programs' key-tile trips are the tiles that the lengths give; their
    wait values are minimal and the simulations are the oracle's."""
    lengths, heads = [300, 1, 257, 640], 3
    sg = example.sg
    assert example.walk(300) == [1, 2, 3] and example.walk(1) == [1] and example.walk(256) == [1, 2]
    h, counts, free, barrier = example.schedule(lengths, heads)
    assert counts == [0, 0]
    batch = workloads.concat([example.program(x, heads, i) for i, x in enumerate(lengths)])
    tiles = sum(sum(example.walk(x)) for x in lengths) * heads
    rows = sum(len(example.walk(x)) for x in lengths) * heads
    assert h.sizes.n_instances == 9 * tiles + 3 * rows
    thr = oracle.thresholds(batch, sg.THR_PERLOOP)
    for got, variant in ((free, sg.SIM_BARRIER_FREE), (barrier, sg.SIM_BARRIER)):
        assert np.array_equal(got, oracle.simulate(batch, thr, sg.THR_PERLOOP, variant).makespan)
    h.close()


def test_main_prints(example, capsys):
    example.main([200, 3], heads=4, kv_heads=2, dim=64)
    out = capsys.readouterr().out
    assert "unsafe 0, over-synchronised 0" in out and "200 tokens" in out
