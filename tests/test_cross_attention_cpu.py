"""Plans of attention to another sequence's states without a GPU: refusals, and
work lists that cover every pair of tiles of a sequence exactly once."""
import ctypes
import random

import numpy as np
import pytest

from tests.test_attention_cpu import desc


@pytest.fixture(scope="module")
def sg():
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


@pytest.mark.parametrize("bad,status", [
    (dict(q=[-1], k=[1]), "ERR_ARG"), (dict(q=[1], k=[-1]), "ERR_ARG"), (dict(q=[1], k=[1], heads=4, kv=3), "ERR_ARG"),
    (dict(q=[1], k=[1], dim=20), "ERR_ARG"), (dict(q=[2, 2], k=[2, 2], q_start=[0, 1]), "ERR_MALFORMED"),
    (dict(q=[2, 2], k=[2, 2], k_start=[0, 1], train=1), "ERR_MALFORMED"), (dict(q=[2], k=[2], k_start=[(1 << 31) - 2]), "ERR_OVERFLOW")], ids=str)
def test_refused(sg, bad, status):
    out = ctypes.c_void_p(1)
    assert sg.lib().sync_cross_attn_plan(ctypes.byref(desc(sg, **bad)), 0, ctypes.byref(out)) == getattr(sg, status)
    assert not out.value
    assert sg.lib().sync_cross_attn_plan(None, 0, ctypes.byref(out)) == sg.ERR_ARG


def work(sg, d, which, width, sms):
    f = sg.lib().syncgb_cross_attn_work
    f.restype = ctypes.c_int64
    f.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_int64]
    n = f(ctypes.byref(d), sms, which, None, 0)
    assert n >= 0
    out = np.zeros((n, width), dtype=np.int64)
    assert f(ctypes.byref(d), sms, which, out.ctypes.data, n) == n
    return out


def batches():
    r = random.Random(6)
    for rep in range(80):
        n = r.randint(1, 6)
        q = [1 if rep % 3 == 0 else r.choice([0, r.randint(1, 2000)]) for _ in range(n)]
        k = [r.choice([0, r.randint(1, 9000), r.randint(1, 300)]) for _ in q]
        kv = r.choice([1, 2, 8])
        yield q, k, kv * r.choice([1, 3, 5, 16]), kv, r.choice([1, 4, 152])


def test_forward_items_meet_every_key_once(sg):
    for q, k, heads, kv, sms in batches():
        g = heads // kv
        rows = work(sg, desc(sg, q, k, heads, kv), 0, 12, sms)
        seen = {}
        for _, q_row, k_row, head, packed, r0, r1, n0, n1, vis, keys, _ in rows:
            s = max(i for i in range(len(q)) if sum(q[:i]) <= q_row and q[i])
            first, left = k_row - sum(k[:s]), sum(k[:s]) + k[s] - k_row
            assert keys == left and vis >= left         # no key of the piece is hidden
            assert all(n * 128 < left + 128 for n, r in ((n0, r0), (n1, r1)) if n)
            for t, (r_, n_) in enumerate(((r0, n0), (r1, n1))):
                per = 128 // g if packed else 128
                for i in range(r_):
                    for h in range(head, head + (g if packed else 1)):
                        seen.setdefault((q_row + t * per + i, h), []).append((first // 128, first // 128 + n_))
        for s in range(len(q)):
            for i in range(sum(q[:s]), sum(q[:s]) + q[s]):
                for h in range(heads):
                    at = 0
                    for a, b in sorted(seen[(i, h)]):
                        assert a == at
                        at = b
                    assert at == -(-k[s] // 128)
        assert len(seen) == sum(q) * heads


def test_gradient_tiles_meet_all_of_the_other_side(sg):
    for q, k, heads, kv, sms in batches():
        d = desc(sg, q, k, heads, kv, train=1)
        for which, mine, others, h in ((2, q, k, heads), (3, k, q, kv)):
            rows = work(sg, d, which, 8, sms)
            assert len(rows) == h * sum(-(-x // 128) for x in mine)
            assert len({(r[1 if which == 2 else 2], r[3]) for r in rows}) == len(rows)
            for _, q_row, k_row, _, n, left_q, left_k, vis in rows:
                row = q_row if which == 2 else k_row
                s = max(i for i in range(len(q)) if sum(mine[:i]) <= row and mine[i])
                assert n == -(-others[s] // 128)
                if which == 2:
                    assert k_row == sum(k[:s]) and left_k == k[s] == vis and left_q == sum(q[:s + 1]) - q_row
                else:
                    assert q_row == sum(q[:s]) and left_q == q[s] and left_k == sum(k[:s + 1]) - k_row and vis >= 128
