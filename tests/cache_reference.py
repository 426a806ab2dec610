"""The paged cache and the attention that reads it from their definitions, with
bounds on what rounding may do.

Attention, for each entry of an output row with weights w (64 bits), values v:

  weights   16 bits: rounded once to the type (u); 4 bits: once to float16 and
            once more with the value's scale (2 * 2^-11)
  small     a weight's relative error from 32-bit arithmetic: the score's (a sum
            of at most 128 products, each addition off by 2^-23 of the sum of
            sizes; in 4 bits a code and what is taken off it are at most 15 and 8
            where the value is up to 7), its product with the scale (2^-22 of it),
            and 2^-18 for exponentials, rescaling and joining pieces
  adding    n / 16 + 20 additions of 2^-23 of the sum of sizes each
  tiny      what a weight below the normal range is off by whatever its size:
            2^-25 in float16 relative to the largest weight (twice that, and the
            same for its product with the scale, in 4 bits), flushed below 2^-126
            in bfloat16
  result    rounded once (u |o|)
"""
import math

import torch

from tests import attn_reference as ref

U, TINY = ref.U, ref.TINY


def places(table, page, n):
    """(page numbers, offsets) of a sequence's first n tokens."""
    pos = torch.arange(n, device=table.device)
    return table[pos // page].long(), pos % page


def decoded(codes, scale):
    """The values of rows of 4-bit codes in 64 bits, entry by entry."""
    dim = codes.shape[-1] * 2
    d = torch.arange(dim, device=codes.device)
    w, c, e = d // 32, d // 8 % 4, d % 8
    byte = 4 * (dim // 32 * c + w) + e // 2
    n = codes[..., byte].int() >> (4 * (e % 2)) & 15
    return (n - 8).double() * scale.double()[..., w]


def encoded(x):
    """Codes and scales of float32 rows: what a row is written as."""
    g = x.shape[-1] // 32
    y = x.unflatten(-1, (g, 32))
    top = y.abs().amax(-1)
    top = torch.where(torch.isfinite(y).all(-1), top, math.nan)
    scale = torch.clamp(top / torch.full_like(top, 7.0), max=65504.0).half()
    by = scale.float()[..., None]
    n = torch.where(by > 0, y / by, 0.0).round().clamp(-7, 7)
    n = torch.where(torch.isnan(n), 0.0, n).int() + 8
    word = (n.unflatten(-1, (4, 8)) << (4 * torch.arange(8, device=x.device, dtype=torch.int32))).sum(-1)   # [.., g, 4]
    word = word.transpose(-1, -2).flatten(-2)                                                              # word g c + w
    return torch.stack([word >> (8 * b) & 255 for b in range(4)], -1).flatten(-2).to(torch.uint8), scale


def values(cache, name, table, n):
    """[n, kv_heads, dim] of a sequence in 64 bits, and the size of a code's step
    (0 in 16 bits)."""
    p, o = places(table, cache.page, n)
    rows = getattr(cache, name)[p, :, o]
    if cache.bits == 16:
        return rows.double(), torch.zeros_like(rows, dtype=torch.float64)
    scale = getattr(cache, name + "_scale")[p, :, o]
    return decoded(rows, scale), scale.double().repeat_interleave(32, -1)


def attention(cache, q, table, lens, starts, scale):
    """{o, o_tol, o_var, lse, lse_tol}; rows of no sequence are NaN."""
    heads, kv, bits = q.shape[1], cache.kv_heads, cache.bits
    g, u = heads // kv, U[q.dtype]
    up, tiny = (u, TINY[q.dtype]) if bits == 16 else (2 * 2.0 ** -11, 4 * 2.0 ** -25)
    r = {x: torch.full(q.shape, math.nan, dtype=torch.float64, device=q.device) for x in ("o", "o_tol", "o_var")}
    r.update({x: torch.full((heads, q.shape[0]), math.nan, dtype=torch.float64, device=q.device) for x in ("lse", "lse_tol")})
    starts = list(range(len(lens) + 1)) if starts is None else starts
    for s, m in enumerate(lens):
        a, b = starts[s], starts[s + 1]
        n = b - a
        if n == 0:
            continue
        m = max(m, 0)
        k, ks = values(cache, "k", table[s], m)
        v, vs = values(cache, "v", table[s], m)
        for h in range(heads):
            x, kk, vv = q[a:b, h].double(), k[:, h // g], v[:, h // g]
            e = x @ kk.T * scale
            size = x.abs() @ (kk.abs() + 16 * ks[:, h // g]).T * scale
            hidden = torch.arange(m, device=q.device) > (m - n + torch.arange(n, device=q.device))[:, None]
            e = e.masked_fill(hidden, -math.inf)
            size = size.masked_fill(hidden, 0.0)
            small = 2.0 ** -18 + (160 * 2.0 ** -23) * size.amax(1) if m else torch.full((n,), 2.0 ** -18, dtype=torch.float64, device=q.device)
            lse = torch.logsumexp(e, 1) if m else torch.full((n,), -math.inf, dtype=torch.float64, device=q.device)
            w = torch.exp(e - torch.where(lse == -math.inf, 0.0, lse)[:, None])
            o = w @ vv
            top = w.amax(1)[:, None] if m else torch.zeros(n, 1, dtype=torch.float64, device=q.device)
            seen = (~hidden).sum(1)[:, None]
            tol = (up + small[:, None]) * (w @ vv.abs()) + (m / 16 + 20) * 2.0 ** -23 * (w @ (vv.abs() + 16 * vs[:, h // g]))
            tol = tol + tiny * seen * top * (2 * vv.abs().amax() if m else 0.0) + u * o.abs() + TINY[q.dtype]
            r["o"][a:b, h], r["o_tol"][a:b, h] = o, tol
            r["o_var"][a:b, h] = (up * up * (w * w) @ (vv * vv) + (u * o) ** 2) / 3
            r["lse"][h, a:b], r["lse_tol"][h, a:b] = lse, small + 2.0 ** -19 * (1 + torch.where(lse == -math.inf, 0.0, lse).abs())
    return r


def check(got, want):
    """Every entry within its bound, and the norm of each head's error within
    that of independent roundings (half as much again, and a part in 2^15 of the
    result for what is not a rounding)."""
    o, lse = got
    ref.check(o, want["o"], want["o_tol"], "o")
    if lse is not None:
        ref.check(lse, want["lse"], want["lse_tol"], "lse")
    mine = ~torch.isnan(want["o"][:, 0, 0])
    off = (o.double() - want["o"])[mine].square().sum((0, 2)).sqrt()
    allowed = 1.5 * want["o_var"][mine].sum((0, 2)).sqrt() + 2.0 ** -15 * want["o"][mine].square().sum((0, 2)).sqrt() + TINY[o.dtype]
    if off.numel() and int(mine.sum()) * o.shape[2] >= 256:
        assert bool((off <= allowed).all()), f"norms of the errors {off.tolist()} where {allowed.tolist()} are allowed"
