"""Attention over the paged cache where most weights are far below the largest
and values of a head differ in size: a first token that takes the row, thousands
of others with next to nothing each, groups of channels and single tokens whose
scales are far from the rest.  What the many add together has to survive, in
every group of 32 entries for itself.

Bounds, for an entry of a group with weights w (64 bits) and values v:

  weights   rounded once to the type (2^-11 in float16, 2^-8 in bfloat16), in 4
            bits to float16 before and after their value's scale
  tiny      a weight too small for float16's normal numbers is off by half a step
            of 2^-24 where the largest stands for 2^11 at least: 2^-36 of the largest
            weight; in 4 bits twice that (before and after), times a power of two
            above the group's largest scale and a code of up to 8
  scales    in 4 bits one too small for the same reason is off by 2^-25 of that power
            of two, alike for tokens of equal scale
  result    rounded once

and the norm of a group's errors (rows and entries together) that of independent
roundings, uniform within these bounds, half as much again, with the scales' in full
and 2^-15 of the result for 32-bit arithmetic."""
import math

import pytest
import torch

from tests import cache_reference as ref
from tests.attn_reference import TINY, U
from tests.test_gpu_cache import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


N, PAGE, SEQS = 8192, 64, 300      # 300 sequences share the pages: a warp has whole passes, the first token's with them


def signs(dim):
    return 1.0 - 2.0 * (torch.arange(dim, device="cuda") * 7 % 11 % 2)


def packed_codes(n):
    """[.., dim] codes from -8 to 7 as a cache's bytes hold them (as encoded() lays them out)."""
    g = n.shape[-1] // 32
    word = ((n + 8).int().unflatten(-1, (g, 4, 8)) << (4 * torch.arange(8, device=n.device, dtype=torch.int32))).sum(-1)
    word = word.transpose(-1, -2).flatten(-2)
    return torch.stack([word >> (8 * b) & 255 for b in range(4)], -1).flatten(-2).to(torch.uint8)


def setting(sg, bits, kv, heads, dim, dtype, nats, first_value, groups, tokens, rows=1, seed=1):
    """A cache of N tokens that all sequences read, their queries, and the scale:
    the first token's score is `nats` above the others', which spread by a third.
    groups: sizes of the groups' values; tokens: size of every 2000th token's."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache = sg.sync_kv_cache(N // PAGE, PAGE, kv, dim, dtype, bits=bits)
    shape, s = (N // PAGE, kv, PAGE, dim), signs(dim)
    k = torch.randint(-7, 8, shape, generator=g, device="cuda").float()
    v = torch.randint(2, 8, shape, generator=g, device="cuda") * s
    k[0, :, 0] = 7 * s
    k_scale = torch.full(shape[:3] + (dim // 32,), 0.3 / 4.3, device="cuda")
    k_scale[0, :, 0] = nats / (7 * math.sqrt(dim))
    v_scale = torch.tensor(groups, device="cuda")[torch.arange(dim // 32, device="cuda") % len(groups)].expand_as(k_scale).clone()
    t = (torch.arange(N, device="cuda") % 2000 == 1999).view(N // PAGE, 1, PAGE, 1)
    v_scale = torch.where(t, v_scale * tokens, v_scale)
    v_scale[0, :, 0] *= first_value
    if bits == 4:
        cache.k.copy_(packed_codes(k))
        cache.v.copy_(packed_codes(v))
        cache.k_scale.copy_(k_scale)
        cache.v_scale.copy_(v_scale)
    else:
        cache.k.copy_(k * k_scale.repeat_interleave(32, -1))
        cache.v.copy_(v * v_scale.repeat_interleave(32, -1))
    q = (s + 0.05 * torch.randn((SEQS * rows, heads, dim), generator=g, device="cuda")).to(dtype)
    table = torch.arange(N // PAGE, device="cuda", dtype=torch.int32).expand(SEQS, -1).contiguous()
    return cache, q, table


def check_groups(cache, q, o, rows):
    heads, kv, dim, dtype = q.shape[1], cache.kv_heads, cache.head_dim, q.dtype
    at = torch.arange(N // PAGE, device="cuda", dtype=torch.int32)
    k, _ = ref.values(cache, "k", at, N)
    v, step = ref.values(cache, "v", at, N)
    u = U[dtype]
    for first in (0, 137 * rows, (SEQS - 1) * rows):
        x, got = q[first:first + rows].double(), o[first:first + rows].double()
        for kh in range(kv):
            hs = slice(kh * (heads // kv), (kh + 1) * (heads // kv))
            e = torch.einsum("rhd,nd->rhn", x[:, hs], k[:, kh]) * dim ** -0.5
            e = e.masked_fill((torch.arange(N, device="cuda") > N - rows + torch.arange(rows, device="cuda")[:, None])[:, None], -math.inf)
            w = torch.softmax(e, -1)
            want = w @ v[:, kh]
            if cache.bits == 4:
                up, most = math.sqrt(2) * 2.0 ** -11, 16 * step[:, kh].amax(0)
                absolute = 2 * N * (w.amax(-1, keepdim=True) * 2.0 ** -36 * most).square()
            else:
                up, most, tiny = u, torch.zeros_like(step[0, kh]), 0.0 if dtype is torch.bfloat16 else 2.0 ** -36
                absolute = (w.amax(-1, keepdim=True) * tiny).square() * v[:, kh].square().sum(0)
            var = (up * up * (w * w) @ v[:, kh].square() + absolute + (u * want).square()) / 3 + TINY[dtype] ** 2
            off = (got[:, hs] - want).unflatten(-1, (-1, 32)).square().sum((0, -1)).sqrt()
            norm = want.unflatten(-1, (-1, 32)).square().sum((0, -1)).sqrt()
            scales = 2.0 ** -25 * (most.unflatten(-1, (-1, 32)).square().sum(-1) * rows).sqrt()
            allowed = 1.5 * var.unflatten(-1, (-1, 32)).sum((0, -1)).sqrt() + scales + 2.0 ** -15 * norm
            assert bool((off <= allowed).all()), f"errors {(off / norm).tolist()} of the groups' norms where {(allowed / norm).tolist()} are allowed"


DTYPE = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])


@DTYPE
@pytest.mark.parametrize("nats", [10.0, 12.0, 14.0])
@pytest.mark.parametrize("groups,tokens", [((1.0, 1.0, 0.5, 1.0 / 32), 1.0), ((1.0, 1.0 / 128), 1.0), ((1.0,), 200.0), ((1.0, 1.0 / 32), 200.0)], ids=str)
def test_small_weights_in_4_bits(sg, groups, tokens, nats, dtype):
    for heads, kv, dim, rows in ((32, 8, 128, 1), (12, 1, 128, 3), (8, 8, 64, 1), (8, 8, 96, 1)):
        cache, q, table = setting(sg, 4, kv, heads, dim, dtype, nats, 0.05, groups, tokens, rows)
        starts = None if rows == 1 else i32([rows * s for s in range(SEQS + 1)])
        o = sg.sync_cache_attn(cache, q, table, i32([N] * SEQS), starts, max_new=rows)
        check_groups(cache, q, o, rows)


@pytest.mark.parametrize("tokens", [1.0, 3e4])
def test_groups_of_very_different_size(sg, tokens):
    """Scales from one end of float16's range to the other, beside one another in a row."""
    cache, q, table = setting(sg, 4, 8, 32, 128, torch.bfloat16, 6.0, 1.0, (1.3, 1.3 * 2.0 ** -14, 2.0 ** -7, 1.7), tokens)
    check_groups(cache, q, sg.sync_cache_attn(cache, q, table, i32([N] * SEQS)), 1)


@DTYPE
@pytest.mark.parametrize("nats", [12.0, 17.0])
def test_small_weights_in_16_bits(sg, nats, dtype):
    for heads, kv, dim, rows in ((32, 8, 128, 1), (16, 4, 64, 3)):
        cache, q, table = setting(sg, 16, kv, heads, dim, dtype, nats, 1e-3, (1.0,), 1.0, rows)
        starts = None if rows == 1 else i32([rows * s for s in range(SEQS + 1)])
        o = sg.sync_cache_attn(cache, q, table, i32([N] * SEQS), starts, max_new=rows)
        check_groups(cache, q, o, rows)
