"""The attention block's operators without a GPU: their C calls refuse bad
arguments before any device work, and a plan's work lists cover every pair of
tiles exactly once, whatever the lengths."""
import ctypes
import random

import numpy as np
import pytest


@pytest.fixture(scope="module")
def sg():
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


def desc(sg, q, k, heads=4, kv=2, dim=64, dtype=0, train=0, q_start=None, k_start=None):
    d = sg.attention.AttnDesc()
    keep = [np.array(q, dtype=np.int32), np.array(k, dtype=np.int32)]
    d.n_seqs = len(q)
    d.q_len, d.k_len = (a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)) for a in keep)
    for name, v in (("q_start", q_start), ("k_start", k_start)):
        if v is not None:
            keep.append(np.array(v, dtype=np.int64))
            setattr(d, name, keep[-1].ctypes.data_as(ctypes.POINTER(ctypes.c_int64)))
    d.heads, d.kv_heads, d.head_dim, d.dtype, d.train = heads, kv, dim, dtype, train
    d.keep = keep
    return d


def test_null_arguments(sg):
    lib = sg.lib()
    out = ctypes.c_void_p()
    assert lib.sync_attn_plan(None, 0, ctypes.byref(out)) == sg.ERR_ARG
    assert lib.sync_attn_plan(ctypes.byref(desc(sg, [1], [1])), 0, None) == sg.ERR_ARG
    d = desc(sg, [1], [1])
    d.q_len = None
    assert lib.sync_attn_plan(ctypes.byref(d), 0, ctypes.byref(out)) == sg.ERR_ARG
    assert lib.sync_attn_query(None, None) == sg.ERR_ARG
    assert lib.sync_attn_forward(None, None, None, None, 1.0, None, None, None) == sg.ERR_ARG
    assert lib.sync_attn_backward(None, None, None, None, None, None, None, 1.0, None, None, None, None) == sg.ERR_ARG
    assert lib.sync_qk_norm_rope(None, None, None, None) == sg.ERR_ARG
    assert lib.sync_qk_norm_rope_backward(None, None, None, None, None, None, None, None, 0, None) == sg.ERR_ARG
    assert lib.sync_qk_norm_rope_workspace(None, None) == sg.ERR_ARG
    lib.sync_attn_free(None)
    assert "NULL" in lib.sync_last_error().decode()


@pytest.mark.parametrize("bad,status", [
    (dict(q=[-1], k=[1]), "ERR_ARG"), (dict(q=[1], k=[-1]), "ERR_ARG"), (dict(q=[1], k=[1], heads=0), "ERR_ARG"),
    (dict(q=[1], k=[1], heads=4, kv=3), "ERR_ARG"), (dict(q=[1], k=[1], dim=4), "ERR_ARG"), (dict(q=[1], k=[1], dim=136), "ERR_ARG"),
    (dict(q=[1], k=[1], dim=20), "ERR_ARG"), (dict(q=[1], k=[1], dtype=2), "ERR_ARG"), (dict(q=[1], k=[1], dtype=-1), "ERR_ARG"),
    (dict(q=[1], k=[1], q_start=[-1]), "ERR_ARG"), (dict(q=[2, 2], k=[2, 2], q_start=[0, 1]), "ERR_MALFORMED"),
    (dict(q=[2, 2], k=[2, 2], k_start=[0, 1], train=1), "ERR_MALFORMED"),
    (dict(q=[2], k=[2], k_start=[(1 << 31) - 2]), "ERR_OVERFLOW"), (dict(q=[2], k=[2], q_start=[1 << 40]), "ERR_OVERFLOW")], ids=str)
def test_descriptions_refused(sg, bad, status):
    out = ctypes.c_void_p(1)
    assert sg.lib().sync_attn_plan(ctypes.byref(desc(sg, **bad)), 0, ctypes.byref(out)) == getattr(sg, status)
    assert not out.value


@pytest.mark.parametrize("change", [
    dict(dtype=3), dict(heads=0), dict(kv_heads=0), dict(dim=0), dict(dim=7), dict(dim=258), dict(rotated=-2), dict(rotated=66),
    dict(rotated=3), dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf"))], ids=str)
def test_norm_refused(sg, change):
    A = sg.attention
    p = A.NormRope(0, 4, 2, 64, 64, 0, 1e-6, A.Rows(256, 5, 256, 64), A.Rows(256, 5, 128, 64), None, None, 256, 256, 10, None)
    for name, v in change.items():
        setattr(p, name, v)
    n = ctypes.c_int64()
    assert sg.lib().sync_qk_norm_rope_workspace(p, n) == sg.ERR_ARG
    assert sg.lib().sync_qk_norm_rope(p, A.Rows(256, 5, 256, 64), A.Rows(256, 5, 128, 64), None) == sg.ERR_ARG


def work(sg, d, which, width, sms=152):
    f = sg.lib().syncgb_attn_work
    f.restype = ctypes.c_int64
    f.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_int64]
    n = f(ctypes.byref(d), sms, which, None, 0)
    assert n >= 0
    out = np.zeros((n, width), dtype=np.int64)
    assert f(ctypes.byref(d), sms, which, out.ctypes.data, n) == n
    return out


def batches():
    r = random.Random(5)
    for rep in range(120):
        n = r.randint(1, 40 if rep % 6 == 0 else 6)
        kind = rep % 4
        q = [1 if kind == 0 else r.randint(0, 4) if kind == 1 else r.randint(0, 2000) for _ in range(n)]
        k = [r.randint(0, 2000) if kind == 3 else x + r.choice([0, r.randint(0, 9000)]) for x in q]
        kv = r.choice([1, 2, 8])
        yield q, k, kv * r.choice([1, 3, 4, 5, 16, 200 if rep % 11 == 0 else 2]), kv, r.choice([1, 4, 152])
    yield [], [], 4, 2, 152
    yield [8192], [8192], 32, 32, 152


def test_forward_work_covers_every_tile_once(sg):
    for q, k, heads, kv, sms in batches():
        g = heads // kv
        d = desc(sg, q, k, heads, kv)
        items, splits = work(sg, d, 0, 12, sms), work(sg, d, 1, 7, sms)
        assert np.all(np.diff(items[:, 0]) >= 0) and (len(items) == 0 or items[-1, 0] < sms)
        pieces = {}
        for row in items:
            pieces.setdefault((row[1], row[3]), []).append(row)
        slots = sorted(int(x) for x in items[:, 11] if x >= 0)
        assert slots == list(range(len(slots)))
        split = {(s[0], s[1]): s for s in splits}
        expected = 0
        q0 = k0 = 0
        for lq, lk in zip(q, k):
            per = 128 // g if 1 < g <= 128 and -(-lq // (128 // g)) < g * -(-lq // 128) else 128
            packed = per != 128 or (1 < g <= 128 and lq > 0 and -(-lq // (128 // g)) < g * -(-lq // 128))
            for h in range(0, heads, g if packed else 1):
                for a in range(0, lq, 2 * per):
                    expected += 1
                    rows = sorted(pieces[(q0 + a, h)], key=lambda x: x[2])
                    assert all(x[4] == packed for x in rows)
                    n = [0, 0]
                    at = 0
                    for i, x in enumerate(rows):
                        assert x[2] == k0 + 128 * at and x[9] == a + lk - lq + 1 - 128 * at and x[10] == lk - 128 * at
                        assert (x[11] >= 0) == (len(rows) > 1) and (len(rows) == 1 or x[11] == rows[0][11] + i)
                        assert len(rows) == 1 or max(x[7], x[8]) > 0
                        n[0] += x[7]
                        n[1] += x[8]
                        at += max(x[7], x[8])
                    for t in range(2):
                        have = max(0, min(per, lq - a - t * per))
                        seen = max(0, a + t * per + have + lk - lq) if have else 0
                        assert rows[0][5 + t] == have and n[t] == -(-seen // 128)
                    if len(rows) > 1:
                        s = split.pop((q0 + a, h))
                        assert s[2] == packed and s[5] == rows[0][11] and s[6] == len(rows) and list(s[3:5]) == list(rows[0][5:7])
            q0 += lq
            k0 += lk
        assert expected == len(pieces) and not split


def test_forward_work_is_balanced(sg):
    """A block's share is at most 1/8 (and an item's own cost) above the mean."""
    for q, k, heads, kv in (([1] * 64, [random.Random(i).randint(1, 8192) for i in range(64)], 32, 8), ([8192], [8192], 32, 32),
                            ([300, 1500, 90], [4300, 1500, 4000], 32, 4)):
        items = work(sg, desc(sg, q, k, heads, kv, 128), 0, 12)
        cost = np.zeros(152)
        np.add.at(cost, items[:, 0], items[:, 7] + items[:, 8] + 4)
        assert cost.max() <= cost.mean() * 1.125 + 6


def test_gradient_work_covers_every_tile_once(sg):
    for q, k, heads, kv, sms in batches():
        d = desc(sg, q, k, heads, kv, train=1)
        by_query, by_key = ({(x[1] if which == 2 else x[2], x[3]): x for x in work(sg, d, which, 8, sms)} for which in (2, 3))
        q0 = k0 = 0
        for lq, lk in zip(q, k):
            off = lk - lq
            for h in range(heads):
                for a in range(0, lq, 128):
                    x = by_query.pop((q0 + a, h))
                    seen = max(0, min(a + 128, lq) + off)
                    assert x[2] == k0 and x[4] == -(-seen // 128) and x[5] == lq - a and x[6] == lk and x[7] == a + off + 1
            for h in range(kv):
                for b in range(0, lk, 128):
                    x = by_key.pop((k0 + b, h))
                    first = max(0, b - off) // 128                  # the first tile with a query that sees key b
                    n = max(0, -(-lq // 128) - first)
                    assert x[4] == n and x[6] == lk - b
                    if n:
                        assert x[1] == q0 + 128 * first and x[5] == lq - 128 * first and x[7] == 128 * first + off + 1 - b
            q0 += lq
            k0 += lk
        assert not by_query and not by_key
