"""Attention over packed sequences, and head norms with the rotation, from their
definitions in 64 bits, with bounds on what rounding may do to each entry.

The bounds follow the operators' documented precision.  u is half a unit in
the last place of 1 in the tensors' type (2^-8 for bfloat16, 2^-11 for
float16), the largest relative error of one rounding to it:

  o    weights rounded once (u sum w|v|), the result rounded once (u |o|)
  dv   weights rounded once, the result rounded once
  ds   rounded once (u |ds|); the row sum delta = sum o do uses the rounded o,
       whose error times |do| enters every ds of the row with its weight
  dq   = scale ds k, dk = scale ds^T q: the errors of ds summed with |k|, |q|,
       and the result rounded once

SMALL covers the 32-bit arithmetic: scores of at most 128 products (an error
below 128 * 2^-24 * sum |q k| scale, which is a relative error of the weight),
exp2 to 2^-22 and sums.  TINY is what a value below the normal range may be
off by whatever its size: 2^-25 for float16 (half its smallest step), 2^-126
for bfloat16 and 32 bits (flushed to zero).
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


def visible(n, m, device):
    """Query i of n sees key j of m: j <= i + m - n."""
    i = torch.arange(n, device=device)[:, None]
    return torch.arange(m, device=device)[None] <= i + (m - n)


def head(q, k, v, scale, do=None):
    """One head of one sequence in 64 bits: a dict of o, lse and, with do, dq,
    dk, dv, and the bound of each under `name + "_tol"` given the type of q."""
    u, tiny = U[q.dtype], TINY[q.dtype]
    q, k, v = q.double(), k.double(), v.double()
    n, m = q.shape[0], k.shape[0]
    s = (q @ k.T) * scale
    small = 2.0 ** -20 + 128 * 2.0 ** -24 * float(((q.abs() @ k.abs().T) * scale).max()) if n and m else 2.0 ** -20
    s = s.masked_fill(~visible(n, m, q.device), -math.inf)
    lse = torch.logsumexp(s, 1) if m else torch.full((n,), -math.inf, dtype=torch.float64, device=q.device)
    w = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None])
    o = w @ v
    wv = w @ v.abs()
    # the largest unnormalised weight of a row is at least 1, so tiny is relative to it
    o_err = (u + small) * wv + tiny * m * (v.abs().amax() if m else 0.0)
    r = {"o": o, "o_tol": o_err + u * o.abs() + tiny, "lse": lse, "lse_tol": small + 2.0 ** -20 * (1 + lse.abs())}
    if do is None:
        return r
    do = do.double()
    dp = do @ v.T
    delta = (do * o).sum(1, keepdim=True)
    delta_err = ((o_err + u * o.abs()) * do.abs()).sum(1, keepdim=True) + 2.0 ** -18 * (do.abs() @ v.abs().T).amax(1, keepdim=True) if m else delta
    ds = w * (dp - delta)
    # a weight below 2^-126 is zero
    ds_err = (u + 2 * small) * ds.abs() + w * delta_err + tiny + 2.0 ** -126 * (dp - delta).abs() + small * w * (do.abs() @ v.abs().T)
    dv, dq, dk = w.T @ do, ds @ k * scale, ds.T @ q * scale
    r["dv"], r["dv_tol"] = dv, (u + 2 * small) * (w.T @ do.abs()) + tiny * do.abs().sum(0) + u * dv.abs() + tiny
    r["dq"], r["dq_tol"] = dq, (ds_err @ k.abs()) * scale + u * dq.abs() + tiny
    r["dk"], r["dk_tol"] = dk, (ds_err.T @ q.abs()) * scale + u * dk.abs() + tiny
    return r


def packed(q, k, v, q_lens, k_lens, q_starts, k_starts, scale, do=None):
    """Every head of every sequence: {name: 64-bit tensor shaped as the
    operator's}; rows of no sequence are NaN.  Bounds of sums over query heads
    add up (each head's own, though the sum is rounded once)."""
    heads, kv = q.shape[1], k.shape[1]
    g = heads // kv

    def nan(t):
        return torch.full(t.shape, math.nan, dtype=torch.float64, device=q.device)
    names = ["o"] + (["dq", "dk", "dv"] if do is not None else [])
    shape = {"o": q, "dq": q, "dk": k, "dv": k}
    r = {x + e: nan(shape[x]) for x in names for e in ("", "_tol")}
    for e in ("lse", "lse_tol"):
        r[e] = torch.full((heads, q.shape[0]), math.nan, dtype=torch.float64, device=q.device)
    for n, m, a, b in zip(q_lens, k_lens, q_starts, k_starts):
        for x in names:
            if x in ("dk", "dv"):
                r[x][b:b + m] = 0
                r[x + "_tol"][b:b + m] = 0
        for h in range(heads):
            one = head(q[a:a + n, h], k[b:b + m, h // g], v[b:b + m, h // g], scale, None if do is None else do[a:a + n, h])
            for x in names:
                for e in ("", "_tol"):
                    if x in ("dk", "dv"):
                        r[x + e][b:b + m, h // g] += one[x + e]
                    else:
                        r[x + e][a:a + n, h] = one[x + e]
            for e in ("lse", "lse_tol"):
                r[e][h, a:a + n] = one[e]
    return r


def check(got, want, tol, name):
    """Every entry of a sequence within its bound; the same infinities."""
    mine = ~torch.isnan(want)
    g, w, t = got.double()[mine], want[mine], tol[mine]
    inf = torch.isinf(w)
    assert torch.equal(g[inf], w[inf]), f"{name}: infinities differ"
    off = (g - w).abs()[~inf]
    t = t[~inf]
    bad = ~(off <= t)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} entries off, the worst by {float(off[bad].max()):.3g} where {float(t[bad][off[bad].argmax()]):.3g} is allowed"


def norm_rope(x, w, cos, sin, positions, eps, interleaved, dy=None):
    """Norm and rotation of one tensor in 64 bits; with dy its gradient and the
    weights' ([dim], summed)."""
    half = cos.shape[1]
    x = x.double()
    w = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if w is None else w.double()
    c, s = cos.double()[positions.long()][:, None], sin.double()[positions.long()][:, None]
    one = torch.arange(half, device=x.device) * (2 if interleaved else 1)
    two = one + (1 if interleaved else half)

    def turn(y, way):
        z = y.clone()
        z[..., one] = y[..., one] * c - way * y[..., two] * s
        z[..., two] = y[..., two] * c + way * y[..., one] * s
        return z
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    if dy is None:
        return turn(x * r * w, 1.0)
    d = turn(dy.double(), -1.0)
    dw = (d * x * r).sum((0, 1))
    dw_abs = (d * x * r).abs().sum((0, 1))
    d = d * w
    return r * (d - x * r * (d * x * r).mean(-1, keepdim=True)), dw, dw_abs
