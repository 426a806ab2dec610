"""Arguments of sync_attn_plan that its binding refuses, without a GPU."""
import pytest
import torch


@pytest.fixture(scope="module")
def sg():
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


@pytest.mark.parametrize("device", ["cpu", torch.device("cpu"), torch.device("meta")], ids=str)
def test_devices(sg, device):
    with pytest.raises(sg.SyncError) as e:
        sg.sync_attn_plan([1], [1], 4, 2, 64, torch.bfloat16, device=device)
    assert e.value.status == sg.ERR_ARG


@pytest.mark.parametrize("change", [dict(q_lens=[1.5]), dict(k_lens=[2.25]), dict(q_starts=[0.5]), dict(k_starts=[1e-3]), dict(q_lens=[float("nan")])], ids=str)
def test_fractions(sg, change):
    args = dict(q_lens=[1], k_lens=[2], q_starts=[0], k_starts=[0])
    args.update(change)
    with pytest.raises(sg.SyncError) as e:
        sg.sync_attn_plan(args["q_lens"], args["k_lens"], 4, 2, 64, torch.bfloat16, q_starts=args["q_starts"], k_starts=args["k_starts"], device=0)
    assert e.value.status == sg.ERR_ARG and "whole" in str(e.value)
