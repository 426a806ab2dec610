"""How far the attention operators may be off as a whole: bounds on the norm of
the error of each output of a head of a sequence, which a wrong factor, a wrong
mask or a missing term exceeds (the bounds of attn_reference.py on single
entries add up every rounding's largest error, and are many times wider).

One rounding changes a value by a factor 1 + e with |e| <= u (attn_reference's),
and the errors of different values are independent, with a standard deviation
of u / sqrt(3) at most (e spread evenly, at the start of a binade).  Taking u
itself, the variances of an output's entries add up from what is rounded on
the way to it:

  o    the weights P before P V, and the result
  delta = sum o do of a row: P by way of do V^T, and the rounded o
  dv   P, and the result
  dq, dk   dS, delta (one error for all keys of a row), and the result; dk
       and dv are summed over the query heads of their key head, then rounded

with `small` of attn_reference for the 32-bit part of a weight and TINY for the
smallest values.  An error's norm is then at most sqrt(1 / 3) of sqrt(sum of
the variances) on average; MARGIN = 2 times that root is 3.4 times as much,
which a sum over hundreds of entries does not reach.  In bfloat16 the bounds
come to about 1% of an output's norm.
"""
import math

import torch

from tests import attn_reference as ref

MARGIN = 2.0


def head(q, k, v, scale, do):
    """One head of one sequence in 64 bits: {name: (value, variance of each
    entry)} of o, dq, dk, dv; for dk and dv without the last rounding."""
    u2, tiny2 = ref.U[q.dtype] ** 2, ref.TINY[q.dtype] ** 2
    q, k, v, do = (x.double() for x in (q, k, v, do))
    n, m = q.shape[0], k.shape[0]
    one = ref.visible(n, m, q.device)
    s = ((q @ k.T) * scale).masked_fill(~one, -math.inf)
    small2 = (2.0 ** -20 + 128 * 2.0 ** -24 * float(((q.abs() @ k.abs().T) * scale).max()) if n and m else 0.0) ** 2
    w = torch.exp(s - torch.logsumexp(s, 1, keepdim=True)).nan_to_num(0.0)       # a row that sees nothing: no weights
    o, dp = w @ v, do @ v.T
    delta = (do * o).sum(1, keepdim=True)
    ds = w * (dp - delta)
    w_var = (u2 + small2) * w.square() + tiny2 * one
    ds_var = (u2 + 2 * small2) * ds.square() + (tiny2 + 2.0 ** -40 * (w * (do.abs() @ v.abs().T)).square()) * one
    o_var = w_var @ v.square()
    delta_var = (w_var * dp.square()).sum(1, keepdim=True) + u2 * (o * do).square().sum(1, keepdim=True)
    dq = ds @ k * scale
    return {"o": (o, o_var + u2 * o.square() + tiny2),
            "dq": (dq, scale ** 2 * (ds_var @ k.square() + (w @ k).square() * delta_var) + u2 * dq.square() + tiny2),
            "dk": (ds.T @ q * scale, scale ** 2 * (ds_var.T @ q.square() + w.square().T @ (q.square() * delta_var))),
            "dv": (w.T @ do, w_var.T @ do.square())}


def check(got, q, k, v, do, q_lens, k_lens, scale):
    """Every (o, dq, dk, dv) of a packed batch, head by head; an AssertionError
    names the outputs that are off.  Returns the largest share of a bound."""
    u2, tiny2 = ref.U[q.dtype] ** 2, ref.TINY[q.dtype] ** 2
    group = q.shape[1] // k.shape[1]
    got = dict(zip(("o", "dq", "dk", "dv"), got))
    off, most = [], 0.0
    a = b = 0

    def compare(name, i, h, mine, value, var):
        nonlocal most
        error, bound = float((mine.double() - value).norm()), MARGIN * math.sqrt(float(var.sum()))
        if not error <= bound:
            off.append((name, i, h, error, bound, float(value.norm())))
        elif bound:
            most = max(most, error / bound)
    for i, (n, m) in enumerate(zip(q_lens, k_lens)):
        for kv in range(k.shape[1]):
            sums = {"dk": [0.0, 0.0], "dv": [0.0, 0.0]}
            for h in range(kv * group, (kv + 1) * group):
                r = head(q[a:a + n, h], k[b:b + m, kv], v[b:b + m, kv], scale, do[a:a + n, h])
                for name in ("o", "dq"):
                    compare(name, i, h, got[name][a:a + n, h], *r[name])
                for name, x in sums.items():
                    x[0], x[1] = x[0] + r[name][0], x[1] + r[name][1]
            for name, (value, var) in sums.items():
                compare(name, i, kv, got[name][b:b + m, kv], value, var + u2 * value.square() + tiny2)
        a, b = a + n, b + m
    assert not off, f"{len(off)} outputs off, such as (name, sequence, head, error, bound, norm) {off[0]}; names {sorted({x[0] for x in off})}"
    return most
