"""A packed batch through an attention block's operators, and the schedule of
its tiles on a multi-engine accelerator.

    python examples/packed_attention.py [length ...]

The block: norm and rotation of the query and key heads, causal attention over
the packed sequences, and the gradients of both.  The walk of its 128-row tiles
-- head > query tile > key tile, the key tiles' trip counts following from the
sequences' lengths -- is then loaded as a batch of programs (one per sequence,
the body of the `attention` configuration), its wait values are evaluated and
checked, and the barrier-free and the barrier scheme are simulated.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_13757_gb300 as sg  # noqa: E402
import workloads  # noqa: E402

TILE = 128
ENGINES = DMA_IN, MATMUL, ACTIVATION, VECTOR, DMA_OUT = range(5)


def angles(positions: int, rotated: int, base: float = 10000.0):
    """cos and sin tables [positions, rotated / 2]."""
    half = rotated // 2
    rate = base ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    a = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * rate
    return a.cos().float(), a.sin().float()


def block(lengths, heads, kv_heads, dim, dtype=torch.bfloat16, seed=0):
    """Forward and backward of the block on random projections; a dict of its tensors."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = sum(lengths)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)
    fused = normal(n, heads + 2 * kv_heads, dim)         # what the projection wrote: queries, keys, values
    q, k, v = fused[:, :heads], fused[:, heads:heads + kv_heads], fused[:, heads + kv_heads:]
    wq, wk = torch.ones(2, dim, device="cuda", dtype=dtype)
    positions = torch.cat([torch.arange(x, dtype=torch.int32) for x in lengths]).cuda() if n else torch.empty(0, dtype=torch.int32, device="cuda")
    cos, sin = angles(max(lengths, default=1), dim)
    norm = (wq, wk, cos, sin, positions)
    qn, kn = sg.sync_qk_norm_rope(q, k, *norm)
    plan = sg.sync_attn_plan(lengths, lengths, heads, kv_heads, dim, dtype, train=True)
    o, lse = sg.sync_attn_forward(plan, qn, kn, v, lse=True)
    do = normal(n, heads, dim)
    dqn, dkn, dv = sg.sync_attn_backward(plan, qn, kn, v, o, lse, do)
    dq, dk, dwq, dwk = sg.sync_qk_norm_rope_backward(q, k, dqn, dkn, *norm)
    return dict(q=q, k=k, v=v, qn=qn, kn=kn, o=o, lse=lse, do=do, dqn=dqn, dkn=dkn, dv=dv, dq=dq, dk=dk, dwq=dwq, dwk=dwk,
                norm=norm, plan=plan)


def walk(length):
    """Key tiles of every query tile of one head."""
    return [-(-min(length, (t + 1) * TILE) // TILE) for t in range(-(-length // TILE))]


def program(length, heads, seed):
    """The tile walk of one sequence as a program: loads, both products, the
    running softmax and the store on five engines, buffers used twice in turn."""
    rng = np.random.default_rng(seed)
    cycles = {DMA_IN: (32, 256), MATMUL: (64, 128), ACTIVATION: (16, 64), VECTOR: (16, 64), DMA_OUT: (32, 256)}
    b = workloads.ProgramBuilder(len(ENGINES))
    trips = walk(length)
    head = b.loop(0, 0, [heads])
    qt = b.loop(head, 0, [len(trips)] * heads)
    kt = b.loop(qt, 1, trips * heads)

    def op(loop, pos, engine):
        lo, hi = cycles[engine]
        return b.instr(loop, pos, engine, int(rng.integers(lo, hi + 1)))
    load_q, norm, store = op(qt, 0, DMA_IN), op(qt, 2, VECTOR), op(qt, 3, DMA_OUT)
    load_k, load_v, qk, top, weights, total, rescale, pv, add = (
        op(kt, i, e) for i, e in enumerate((DMA_IN, DMA_IN, MATMUL, VECTOR, ACTIVATION, VECTOR, VECTOR, MATMUL, VECTOR)))
    for p, c, k in ((load_k, qk, 0), (qk, top, 0), (top, weights, 0), (weights, total, 0), (top, rescale, 0), (weights, pv, 0),
                    (load_v, pv, 0), (pv, add, 0), (rescale, add, 0), (top, top, 1), (total, total, 1), (add, add, 1),
                    (qk, load_k, 2), (pv, load_v, 2), (load_q, qk, 0), (add, norm, 0), (total, norm, 0), (norm, store, 0),
                    (qk, load_q, 1), (store, norm, 1)):
        b.dep(p, c, k)
    return b.batch()


def schedule(lengths, heads):
    """(loaded programs, unsafe and over-synchronised pairs, makespans barrier-free, with barriers)."""
    batch = workloads.concat([program(x, heads, i) for i, x in enumerate(lengths) if x])
    h = sg.sync_load_programs(batch)
    thr = sg.sync_eval_thresholds(h, sg.THR_PERLOOP)
    counts, _ = sg.sync_check_minimal(h, sg.THR_PERLOOP, thr)
    spans = [sg.sync_simulate(h, sg.THR_PERLOOP, thr, variant=v).makespan.cpu().numpy()[:batch.n_programs]
             for v in (sg.SIM_BARRIER_FREE, sg.SIM_BARRIER)]
    return h, counts.cpu().tolist(), spans[0], spans[1]


def main(lengths, heads=32, kv_heads=8, dim=128):
    r = block(lengths, heads, kv_heads, dim)
    torch.cuda.synchronize()
    for name in ("o", "dq", "dk", "dv", "dwq", "dwk"):
        print(f"{name:4s} {list(r[name].shape)} rms {float(r[name].float().square().mean().sqrt()):.4f}")
    h, counts, free, barrier = schedule(lengths, heads)
    print(f"{h.sizes.n_programs} programs, {h.sizes.n_instances} instances, {h.sizes.n_pairs} waits; "
          f"unsafe {counts[0]}, over-synchronised {counts[1]}")
    for x, a, b in zip([x for x in lengths if x], free, barrier):
        print(f"  {x:6d} tokens: barrier-free {a} cycles, with barriers {b} ({a / b:.2f})")
    h.close()
    r["plan"].close()


if __name__ == "__main__":
    main([int(x) for x in sys.argv[1:]] or [700, 2050, 130, 1, 513])
