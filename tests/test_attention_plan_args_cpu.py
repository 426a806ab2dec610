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
