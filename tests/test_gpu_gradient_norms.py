"""The attention operators' outputs as a whole, on the GPU: the norm of each
head's error against the bounds of gradient_norms.py."""
import pytest
import torch

from tests import gradient_norms as norms

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as m
    return m


def run_and_check(sg, q_lens, k_lens, heads, kv, dim, dtype, scale=None, gain=1.5, gradient=1.0, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(n, h, std=1.0):
        return (torch.randn((n, h, dim), generator=g, device="cuda") * std).to(dtype)
    q, k, v, do = normal(sum(q_lens), heads, gain), normal(sum(k_lens), kv), normal(sum(k_lens), kv), normal(sum(q_lens), heads, gradient)
    plan = sg.sync_attn_plan(q_lens, k_lens, heads, kv, dim, dtype, train=True)
    o, lse = sg.sync_attn_forward(plan, q, k, v, scale=scale, lse=True)
    got = (o,) + sg.sync_attn_backward(plan, q, k, v, o, lse, do, scale=scale)
    norms.check(got, q, k, v, do, q_lens, k_lens, scale or dim ** -0.5)
    plan.check()
    plan.close()


LENGTHS = {
    "past a tile": ([129, 127, 255, 1], [129, 127, 255, 1]),
    "after earlier keys": ([5, 130, 1, 64], [300, 131, 700, 1000]),
    "fewer keys than queries": ([7, 200, 130], [3, 60, 129]),
    "empty ones": ([0, 5, 4, 0, 9], [5, 0, 4, 0, 131]),
    "short": ([2, 3, 8, 33], [2, 3, 8, 33]),
}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [128, 64, 80])
@pytest.mark.parametrize("lengths", LENGTHS)
def test_lengths(sg, lengths, dim, dtype):
    run_and_check(sg, *LENGTHS[lengths], 4, 2, dim, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("lens,heads,kv", [([2500], 4, 1), ([2048, 700], 16, 1), ([1500], 16, 2), ([900, 1100], 20, 4), ([600], 200, 1), ([300, 7], 256, 2)], ids=str)
def test_long_ones_and_few_key_heads(sg, lens, heads, kv, dtype):
    """Groups of more heads than a tile has rows among them."""
    run_and_check(sg, lens, lens, heads, kv, 64, dtype)


@pytest.mark.parametrize("gradient", [1e-4, 1e-3, 30.0])
def test_small_and_large_gradients(sg, gradient):
    """In float16 dS keeps fewer bits where it is small: steps of 2^-24."""
    run_and_check(sg, [500, 33], [500, 33], 4, 2, 64, torch.float16, gradient=gradient)
    run_and_check(sg, [500, 33], [500, 33], 4, 2, 64, torch.bfloat16, gradient=gradient)


def test_scales(sg):
    run_and_check(sg, [200], [333], 4, 2, 128, torch.bfloat16, scale=0.2)
    run_and_check(sg, [200], [333], 4, 2, 128, torch.float16, scale=1e-3)
