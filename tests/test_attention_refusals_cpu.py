"""Arguments that a kernel could not use, refused by the C calls before any
device work."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def sg():
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


def description(sg, dtype=0):
    R = sg.attention.Rows
    return sg.attention.NormRope(dtype, 4, 2, 64, 64, 0, 1e-6, R(256, 5, 256, 64), R(256, 5, 128, 64), 256, 256, 256, 256, 10, 256)


def forward(sg, p, q_out=(256, 5, 256, 64), k_out=(256, 5, 128, 64)):
    R = sg.attention.Rows
    return sg.lib().sync_qk_norm_rope(p, R(*q_out), R(*k_out), None)


def backward(sg, p, dq=(256, 5, 256, 64), dk=(256, 5, 128, 64), dwq=256, dwk=256):
    R = sg.attention.Rows
    return sg.lib().sync_qk_norm_rope_backward(p, R(256, 5, 256, 64), R(256, 5, 128, 64), R(*dq), R(*dk), dwq, dwk, 256, 1 << 30, None)


@pytest.mark.parametrize("field,address,dtype", [
    ("q_weight", 257, 0), ("k_weight", 257, 1), ("q_weight", 258, 2), ("k_weight", 258, 2), ("cos", 258, 0), ("sin", 257, 0), ("positions", 258, 0)])
def test_pointers_off_their_type(sg, field, address, dtype):
    p = description(sg, dtype)
    setattr(p, field, address)
    for call in (forward, backward):
        assert call(sg, p) == sg.ERR_ARG
        assert field in sg.lib().sync_last_error().decode()


@pytest.mark.parametrize("name,address,dtype", [("dwq", 257, 0), ("dwk", 258, 2)])
def test_weight_gradients_off_their_type(sg, name, address, dtype):
    assert backward(sg, description(sg, dtype), **{name: address}) == sg.ERR_ARG
    assert "aligned" in sg.lib().sync_last_error().decode()


@pytest.mark.parametrize("name,rows", [("q", (256, 5, 0, 64)), ("k", (256, 5, 0, 64)), ("q", (256, 5, 256, 0)), ("k", (256, 5, 128, 0))])
def test_outputs_that_share_memory(sg, name, rows):
    p = description(sg)
    assert forward(sg, p, **{name + "_out": rows}) == sg.ERR_ARG
    assert "share" in sg.lib().sync_last_error().decode()
    assert backward(sg, p, **{"d" + name: rows}) == sg.ERR_ARG
    assert "share" in sg.lib().sync_last_error().decode()
