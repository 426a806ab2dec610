"""The norm bounds on the attention operators' outputs without a GPU: the 64-bit
formulas against difference quotients, outputs with the documented roundings
inside their bounds, and outputs with a mistake outside."""
import math

import pytest
import torch

from tests import attn_reference as ref
from tests import gradient_norms as norms

BATCHES = {
    "two": ([70, 130], [70, 200], 4, 2, 64),
    "one key head": ([300], [300], 16, 1, 64),
    "fewer keys than queries": ([200, 90], [60, 129], 4, 4, 80),
    "long": ([1200], [1200], 4, 1, 64),
    "small": ([1, 3, 33], [5, 3, 40], 4, 2, 128),
}
DTYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])


def made(q_lens, k_lens, heads, kv, dim, dtype, seed=1, gain=1.5):
    g = torch.Generator().manual_seed(seed)

    def normal(n, h, std=1.0):
        return (torch.randn((n, h, dim), generator=g) * std).to(dtype)
    return normal(sum(q_lens), heads, gain), normal(sum(k_lens), kv), normal(sum(k_lens), kv), normal(sum(q_lens), heads)


def emulated(q, k, v, do, q_lens, k_lens, scale, mistake=""):
    """The operators in 64 bits with the documented roundings to the tensors'
    type (P, dS, o, results), and a mistake if one is named."""
    dtype, group = q.dtype, q.shape[1] // k.shape[1]

    def r(x):
        return x.to(dtype).double()
    out = [torch.zeros(x.shape, dtype=torch.float64) for x in (q, q, k, k)]
    a = b = 0
    for n, m in zip(q_lens, k_lens):
        for h in range(q.shape[1]):
            x, y, z, g = q[a:a + n, h].double(), k[b:b + m, h // group].double(), v[b:b + m, h // group].double(), do[a:a + n, h].double()
            seen = torch.arange(m)[None] <= torch.arange(n)[:, None] + (m - n) + (1 if mistake == "one key more" else 0)
            s = (x @ y.T * scale).masked_fill(~seen, -math.inf)
            top = s.amax(1, keepdim=True).nan_to_num(neginf=0.0)
            p = torch.exp(s - top)
            total = p.sum(1, keepdim=True)
            o = r((r(p) @ z) / torch.where(total == 0, 1.0, total))
            w = p / torch.where(total == 0, 1.0, total)
            delta = (o * g).sum(1, keepdim=True)
            if mistake == "no delta":
                delta = 0 * delta
            if mistake == "the next row's delta":
                delta = delta.roll(1, 0)
            ds = r(w * (g @ z.T - delta))
            out[0][a:a + n, h] = o
            out[1][a:a + n, h] = ds @ y * scale
            if mistake == "a head left out" and h == group - 1:
                continue
            out[2][b:b + m, h // group] += ds.T @ x * scale
            out[3][b:b + m, h // group] += r(w).T @ g
        a, b = a + n, b + m
    return [r(x) for x in out]


@DTYPES
@pytest.mark.parametrize("batch", BATCHES)
def test_documented_roundings_pass(batch, dtype):
    q_lens, k_lens, heads, kv, dim = BATCHES[batch]
    x = made(q_lens, k_lens, heads, kv, dim, dtype)
    most = norms.check(emulated(*x, q_lens, k_lens, dim ** -0.5), *x, q_lens, k_lens, dim ** -0.5)
    assert most > 0.05          # the bounds are not wide of what the roundings do


def rejected(outputs, x, q_lens, k_lens, scale):
    """Names of the outputs that are outside their bounds."""
    names = set()
    for i, name in enumerate(("o", "dq", "dk", "dv")):
        good = emulated(*x, q_lens, k_lens, scale)
        good[i] = outputs[i]
        try:
            norms.check(good, *x, q_lens, k_lens, scale)
        except AssertionError:
            names.add(name)
    return names


@DTYPES
@pytest.mark.parametrize("batch", ["two", "one key head", "fewer keys than queries", "long"])
def test_mistakes_are_rejected(batch, dtype):
    q_lens, k_lens, heads, kv, dim = BATCHES[batch]
    x, scale = made(q_lens, k_lens, heads, kv, dim, dtype), dim ** -0.5
    every = {"o", "dq", "dk", "dv"}
    good = emulated(*x, q_lens, k_lens, scale)
    assert rejected([torch.zeros_like(y) for y in good], x, q_lens, k_lens, scale) == every
    assert rejected([0.95 * y for y in good], x, q_lens, k_lens, scale) == every
    assert rejected([-y for y in good], x, q_lens, k_lens, scale) == every
    for mistake, names in (("no delta", {"dq", "dk"}), ("the next row's delta", {"dq", "dk"}), ("one key more", every)):
        assert rejected(emulated(*x, q_lens, k_lens, scale, mistake), x, q_lens, k_lens, scale) == names, mistake
    if heads > kv:
        assert rejected(emulated(*x, q_lens, k_lens, scale, "a head left out"), x, q_lens, k_lens, scale) == {"dk", "dv"}


def test_formulas_against_differences():
    """The 64-bit gradients' product with a direction is the difference quotient
    of the 64-bit forward pass along it (both references of these tests)."""
    q_lens, k_lens, heads, kv, dim = [40, 7, 90], [40, 60, 30], 4, 2, 32
    q, k, v, do = made(q_lens, k_lens, heads, kv, dim, torch.float16)
    scale, a, b = dim ** -0.5, [0, 40, 47], [0, 40, 100]
    want = ref.packed(q, k, v, q_lens, k_lens, a, b, scale, do)

    def loss(t):
        total = 0.0
        for n, m, i, j in zip(q_lens, k_lens, a, b):
            for h in range(heads):
                s = (t[0][i:i + n, h] @ t[1][j:j + m, h // 2].T * scale).masked_fill(~ref.visible(n, m, "cpu"), -math.inf)
                total += float((torch.softmax(s, 1).nan_to_num(0.0) @ t[2][j:j + m, h // 2] * do[i:i + n, h].double()).sum())
        return total
    base = [x.double() for x in (q, k, v)]
    g = torch.Generator().manual_seed(2)
    for i, name in enumerate(("dq", "dk", "dv")):
        way = torch.randn(base[i].shape, generator=g, dtype=torch.float64)
        h = 1e-5
        moved = [[x + (s * h * way if j == i else 0) for j, x in enumerate(base)] for s in (1, -1)]
        quotient = (loss(moved[0]) - loss(moved[1])) / (2 * h)
        assert abs(float((want[name] * way).sum()) - quotient) <= 1e-6 * float((want[name] * way).abs().sum()), name
    for n, m, i, j in zip(q_lens, k_lens, a, b):
        one = norms.head(q[i:i + n, 0], k[j:j + m, 0], v[j:j + m, 0], scale, do[i:i + n, 0])
        two = ref.head(q[i:i + n, 0], k[j:j + m, 0], v[j:j + m, 0], scale, do[i:i + n, 0])
        for name in ("o", "dq", "dk", "dv"):
            assert torch.allclose(one[name][0], two[name], rtol=1e-12, atol=1e-13)
