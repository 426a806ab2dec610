"""The rotation's and the paged cache's calls without a GPU: they refuse bad
arguments before any device work, and the warps of an attention call divide its
list of work without a gap or an overlap, whatever the lengths."""
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


A = 4096      # an aligned address that no call may look at


def rope(sg, **change):
    C, R = sg.cache, sg.attention.Rows
    turn = dict(rotated=64, interleaved=0, n_axes=1, pair_axis=None, cos=A, sin=A, n_positions=10, positions=A, position_stride=5)
    desc = dict(dtype=0, heads=4, kv_heads=2, dim=64, q=R(A, 5, 256, 64), k=R(A, 5, 128, 64))
    for name, v in change.items():
        (turn if name in turn else desc)[name] = v
    p = C.RopeDesc(turn=C.Rotation(**turn), **desc)
    return sg.lib().sync_rope, p, R(A, 5, 256, 64), R(A, 5, 128, 64)


@pytest.mark.parametrize("change", [
    dict(dtype=3), dict(dtype=-1), dict(heads=0), dict(kv_heads=0), dict(dim=7), dict(dim=0), dict(dim=258), dict(rotated=-2), dict(rotated=66),
    dict(rotated=3), dict(n_axes=0), dict(n_axes=5), dict(n_axes=2, positions=None), dict(n_positions=-1), dict(cos=None), dict(sin=None),
    dict(cos=A + 2), dict(sin=A + 1), dict(positions=A + 2), dict(pair_axis=bytes([0] * 31 + [1])), dict(n_axes=3, pair_axis=bytes([3] + [0] * 31))], ids=str)
def test_rotation_refused(sg, change):
    f, p, q, k = rope(sg, **change)
    assert f(p, q, k, None) == sg.ERR_ARG and sg.lib().sync_last_error()
    assert sg.lib().sync_rope_backward(p, q, k, None) == sg.ERR_ARG


def test_rotation_tensors_refused(sg):
    R = sg.attention.Rows
    f, p, q, k = rope(sg)
    assert f(None, q, k, None) == f(p, None, k, None) == f(p, q, None, None) == sg.ERR_ARG
    for bad in (R(A, 4, 256, 64), R(None, 5, 256, 64), R(A + 1, 5, 256, 64), R(A, 5, 0, 64), R(A, 5, 256, 0)):
        assert f(p, bad, k, None) == sg.ERR_ARG
    for name, bad in (("q", R(A, 4, 256, 64)), ("k", R(A, 6, 128, 64)), ("q", R(A + 1, 5, 256, 64)), ("q", R(A, -1, 256, 64))):
        f, p, q, k = rope(sg, **{name: bad})
        assert f(p, q, k, None) == sg.ERR_ARG


def cache(sg, **change):
    d = dict(dtype=0, bits=16, kv_heads=2, head_dim=64, page=16, n_pages=9, k=A, v=A, k_scale=A, v_scale=A)
    return sg.cache.CacheDesc(**{**d, **change})


def seqs(sg, **change):
    d = dict(n_seqs=3, max_pages=4, page_table=A, table_stride=4, lens=A, row_starts=None)
    return sg.cache.CacheSeqs(**{**d, **change})


def calls(sg, c, s, rows=3, heads=4, scale=0.1, max_new=1, work=A, bytes_=1 << 40, q=None, k=None):
    R = sg.attention.Rows
    q, k = q or R(A, rows, 256, 64), k or R(A, rows, 128, 64)
    lib, turn = sg.lib(), None
    return [lib.sync_cache_append(c, s, k, k, heads, q, q, turn, 0, None),
            lib.sync_cache_attn(c, s, heads, q, scale, max_new, q, None, 0, work, bytes_, None)]


@pytest.mark.parametrize("change", [
    dict(dtype=2), dict(dtype=-1), dict(bits=8), dict(bits=0), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=60), dict(head_dim=136),
    dict(bits=4, head_dim=80), dict(bits=4, head_dim=160), dict(page=0), dict(page=8), dict(page=48), dict(page=2048), dict(n_pages=-1),
    dict(n_pages=1 << 28), dict(k=None), dict(v=None), dict(k=A + 8), dict(v=A + 8), dict(bits=4, k_scale=None), dict(bits=4, v_scale=None),
    dict(bits=4, k_scale=A + 8)], ids=str)
def test_cache_refused(sg, change):
    assert calls(sg, cache(sg, **change), seqs(sg)) == [sg.ERR_ARG] * 2
    s = seqs(sg, row_starts=A)
    R = sg.attention.Rows
    assert sg.lib().sync_cache_read(cache(sg, **change), s, R(A, 3, 128, 64), R(A, 3, 128, 64), 0, None) == sg.ERR_ARG


@pytest.mark.parametrize("change", [
    dict(n_seqs=-1), dict(n_seqs=(1 << 20) + 1), dict(max_pages=-1), dict(max_pages=1 << 28), dict(page_table=None), dict(lens=None),
    dict(page_table=A + 2), dict(lens=A + 1), dict(row_starts=A + 2), dict(n_seqs=2), dict(n_seqs=4)], ids=str)
def test_sequences_refused(sg, change):
    assert calls(sg, cache(sg), seqs(sg, **change)) == [sg.ERR_ARG] * 2


def test_tensors_refused(sg):
    R, c, s, lib = sg.attention.Rows, cache(sg), seqs(sg), sg.lib()
    assert calls(sg, c, s, heads=3) == calls(sg, c, s, heads=0) == [sg.ERR_ARG] * 2
    assert calls(sg, None, s) == calls(sg, c, None) == [sg.ERR_ARG] * 2
    # attention alone: 16-byte accesses, its workspace and numbers
    for change in (dict(q=R(A + 8, 3, 256, 64)), dict(q=R(A, 3, 260, 64)), dict(q=R(A, 3, 256, 68)), dict(scale=0.0), dict(scale=float("nan")),
                   dict(scale=-1.0), dict(max_new=0)):
        assert calls(sg, c, s, **change)[1] == sg.ERR_ARG
    long = seqs(sg, max_pages=9)                  # more than 128 tokens: a workspace is needed
    for change in (dict(work=None), dict(work=A + 8)):
        assert calls(sg, c, long, **change)[1] == sg.ERR_ARG
    q, k = R(A, 3, 256, 64), R(A, 3, 128, 64)
    assert lib.sync_cache_append(c, s, None, k, 0, None, None, None, 0, None) == sg.ERR_ARG
    assert lib.sync_cache_append(c, s, k, R(A, 2, 128, 64), 0, None, None, None, 0, None) == sg.ERR_ARG
    assert lib.sync_cache_append(c, s, k, k, 4, q, None, None, 0, None) == sg.ERR_ARG
    assert lib.sync_cache_append(c, s, k, k, 4, q, R(A, 3, 0, 64), None, 0, None) == sg.ERR_ARG
    assert lib.sync_cache_append(c, s, R(A + 1, 3, 128, 64), k, 0, None, None, None, 0, None) == sg.ERR_ARG
    turn = sg.cache.Rotation(66, 0, 1, None, A, A, 10, None, 0)
    assert lib.sync_cache_append(c, s, k, k, 0, None, None, turn, 0, None) == sg.ERR_ARG
    assert lib.sync_cache_read(c, s, k, k, 0, None) == sg.ERR_ARG and b"row_starts" in lib.sync_last_error()
    s = seqs(sg, row_starts=A)
    for bad in (R(A + 8, 3, 128, 64), R(A, 3, 132, 64), R(A, 2, 128, 64), R(A, 3, 0, 64), None):
        assert lib.sync_cache_read(c, s, k, bad, 0, None) == sg.ERR_ARG
    assert lib.sync_cache_attn_workspace(c, 4, 0, ctypes.c_int64()) == sg.ERR_ARG
    assert lib.sync_cache_attn_workspace(c, 5, 1, ctypes.c_int64()) == sg.ERR_ARG
    assert lib.sync_cache_attn_workspace(None, 4, 1, ctypes.c_int64()) == sg.ERR_ARG


def work(sg, lens, starts, rows_all, room, kv, group, rows, tile, warps, whole=0):
    f = sg.lib().syncgb_cache_attn_work
    f.restype = ctypes.c_int64
    f.argtypes = [ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64] + [ctypes.c_int] * 7 + [ctypes.c_void_p, ctypes.c_int64]
    a = np.array(lens, dtype=np.int32)
    b = None if starts is None else np.array(starts, dtype=np.int32)
    args = (len(lens), a.ctypes.data, None if b is None else b.ctypes.data, rows_all, room, kv, group, rows, tile, whole, warps)
    n = f(*args, None, 0)
    out = np.zeros((n, 12), dtype=np.int64)
    assert f(*args, out.ctypes.data, n) == n
    return out


def test_pieces_cover_every_tile_once(sg):
    r = random.Random(3)
    for rep in range(300):
        n = r.choice([0, 1, 2, 5, 40, 300])
        top = r.choice([3, 70, 1000, 20000])
        lens = [r.choice([0, r.randint(0, top), r.randint(0, top // 10 + 1), -1 if rep % 9 == 0 else 5]) for _ in range(n)]
        tokens = [1 if rep % 2 else r.choice([0, 1, 2, 9]) for _ in range(n)]
        starts = None if rep % 2 else [sum(tokens[:i]) for i in range(n + 1)]
        kv, group, rows = r.choice([1, 2, 8]), r.choice([1, 3, 4, 8, 16]), r.choice([8, 16, 32])
        room, warps, tile = r.choice([1 << 20, 640]), r.choice([1, 7, 304, 1824]), r.choice([16, 32])
        got = work(sg, lens, starts, sum(tokens) if starts else n, room, kv, group, rows, tile, warps)
        units = {}
        for x in got:
            units.setdefault((x[1], x[2], x[3]), []).append(x)
        want = 0
        for s in range(n):
            length, bad = min(max(lens[s], 0), room), lens[s] > room
            tiles = -(-length // tile)
            for h in range(kv):
                for first in range(0, tokens[s] * group, rows):
                    want += 1
                    pieces = units[(s, h, first)]
                    assert all(list(x[4:8]) == [tokens[s], (starts or range(n))[s], length, bad] and x[10] == tiles for x in pieces)
                    at = 0
                    for x in pieces:
                        assert x[8] == at and (x[9] > at or tiles == 0)
                        at = x[9]
                    assert at == tiles
                    b = [int(x[0]) for x in pieces]                # warps that follow one another
                    assert b == list(range(b[0], b[0] + len(b))) and all(x[11] == b[-1] for x in pieces)
        assert want == len(units)
        # a warp has at most one piece that began before (its first) and one that it leaves open (its last)
        for b in set(got[:, 0]):
            mine = got[got[:, 0] == b]
            assert all(x[8] == 0 for x in mine[1:]) and all(x[9] == x[10] for x in mine[:-1])


def test_whole_passes(sg):
    """Where no sequence is long, passes are not cut, and warps have equally many."""
    r = random.Random(5)
    for rep in range(60):
        n = r.choice([0, 1, 9, 200])
        lens, tokens = [r.choice([0, r.randint(0, 128)]) for _ in range(n)], [r.choice([0, 1, 1, 5]) for _ in range(n)]
        starts, kv, group, rows, tile = [sum(tokens[:i]) for i in range(n + 1)], r.choice([1, 8]), r.choice([1, 4, 16]), r.choice([8, 32]), r.choice([16, 32])
        got = work(sg, lens, starts, sum(tokens), 128, kv, group, rows, tile, 1216, whole=1)
        want = sorted((s, h, first) for s in range(n) for h in range(kv) for first in range(0, tokens[s] * group, rows))
        assert sorted((x[1], x[2], x[3]) for x in got) == want and all(x[8] == 0 and x[9] == x[10] == -(-lens[x[1]] // tile) for x in got)
        per = np.bincount(got[:, 0], minlength=1)
        assert len(want) == 0 or per.max() <= -(-len(want) // 1216)


def test_runs_are_equal(sg):
    r = random.Random(4)
    lens = [int(np.exp(r.random() * np.log(16000))) for _ in range(128)]
    got = work(sg, lens, None, 128, 1 << 20, 8, 4, 8, 16, 1216)
    cost = np.zeros(1216)
    np.add.at(cost, got[:, 0], got[:, 9] - got[:, 8] + 1)
    assert cost.max() <= cost.mean() + 30


def test_sequences_without_rows_are_passed_over(sg):
    """Runs of empty slots of any length between, before and behind the others."""
    r = random.Random(6)
    for rep in range(200):
        tokens = []
        for _ in range(r.choice([0, 1, 3, 20])):
            tokens += [0] * r.choice([0, 1, 2, 3, 4, 7, 8, 9, 100, 1000]) + [r.choice([1, 2, 5])]
        tokens += [0] * r.choice([0, 1, 50])
        starts, lens = [sum(tokens[:i]) for i in range(len(tokens) + 1)], [r.choice([0, 3, 700]) for _ in tokens]
        for whole in (0, 1) if max(lens, default=0) <= 128 else (0,):
            got = work(sg, lens, starts, sum(tokens), 1 << 20, 2, 4, 8, 16, r.choice([1, 5, 1216]), whole=whole)
            want = {(s, h, f) for s in range(len(tokens)) for h in range(2) for f in range(0, tokens[s] * 4, 8)}
            assert {(x[1], x[2], x[3]) for x in got} == want
            assert sum(x[9] - x[8] for x in got) == sum(-(-lens[s] // 16) for s, _, _ in want)


def test_rows_past_32_bits_refused(sg):
    R, s = sg.attention.Rows, seqs(sg, row_starts=A)
    for rows, heads in ((1 << 28, 16), ((1 << 30) + 1, 2)):
        q = R(A, rows, 64 * heads, 64)
        assert sg.lib().sync_cache_attn(cache(sg), s, heads, q, 0.1, 1, q, None, 0, A, 1 << 40, None) == sg.ERR_ARG
        assert b"2^30" in sg.lib().sync_last_error()
