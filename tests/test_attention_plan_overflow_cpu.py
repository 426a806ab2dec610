"""Plans whose work lists would have more than INT32_MAX items, which is what their
count holds, are refused before anything is laid out."""
import ctypes

import pytest

from tests.test_attention_cpu import desc


@pytest.fixture(scope="module")
def sg():
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


@pytest.mark.parametrize("make", ["sync_attn_plan", "sync_cross_attn_plan"])
@pytest.mark.parametrize("q,k,heads,kv,train,over", [
    (1, 1, 65536, 65536, 0, True),              # 2^31 items of one query (tiles, or passes of few queries)
    (1, 1, 65536, 32768, 0, False),
    (3, 129, 65536, 32768, 1, True),            # two key tiles each
    (300, 1, 32768, 32768, 0, True),            # two items of query tiles each
], ids=str)
def test_lists_past_32_bits(sg, make, q, k, heads, kv, train, over):
    n = 32768
    d = desc(sg, [q] * n, [k] * n, heads, kv, dim=8, train=train)
    out = ctypes.c_void_p(1)
    if over:
        assert getattr(sg.lib(), make)(ctypes.byref(d), 0, ctypes.byref(out)) == sg.ERR_OVERFLOW
        assert b"work items" in sg.lib().sync_last_error() and not out.value
    elif make == "sync_cross_attn_plan":        # one below: goes on to the device, without one here
        status = sg.lib().sync_cross_attn_plan(ctypes.byref(d), 99, ctypes.byref(out))
        assert status == sg.ERR_CUDA and not out.value
