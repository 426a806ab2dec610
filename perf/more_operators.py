"""The measured operators around a cache of keys and values.

  append     new tokens' keys and values into a paged cache, keys (and queries)
             rotated on the way
  piece      the same for the next pieces of prompts, whose whole contexts are
             then read back as packed rows of 16 bits (for attention over them)
  cached     attention of one or a few new tokens per sequence over the cache,
             held in 16 or in 4 bits
  rope       rotation of query and key heads by positions with several axes,
             and its gradient
  cross      attention in which every query sees all keys of its sequence (an
             encoder's states), and its gradient

A case holds plain sizes; lengths follow from them (`lengths`), so the work of
a case does not depend on the seed.  `run` makes one pass: with `own` false in
elementary torch operations in 32 bits, with `own` true through the package.

The cache: tensors [pages, kv_heads, page, dim] of keys and of values, in the
tensors' type or (4 bits) codes [pages, kv_heads, page, dim / 2] of uint8 with
float16 scales [pages, kv_heads, page, dim / 32].  A row of codes is dim / 8
little-endian words; with g = dim / 32, entry 32 w + 8 c + e (c < 4, e < 8) is
bits 4 e .. 4 e + 3 of word g c + w, as its value / scale[w] + 8.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
POSITIONS = 16384


def _cached(name, op, seqs, new, longest, heads, kv_heads, dim, bits, page, dtype, mix):
    """seqs sequences with up to `longest` cached tokens before up to `new` new
    ones each; `mix` picks the lengths."""
    return {"name": name, "op": op, "seqs": seqs, "new": new, "longest": longest, "heads": heads, "kv_heads": kv_heads, "dim": dim, "bits": bits, "page": page, "dtype": dtype, "mix": mix}


def _rope(name, op, total, heads, kv_heads, dim, rotated, axes, interleaved, dtype):
    return {"name": name, "op": op, "total": total, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rotated": rotated, "axes": axes, "interleaved": interleaved, "dtype": dtype}


def _cross(name, op, seqs, queries, keys, heads, kv_heads, dim, dtype, mix):
    """seqs sequences with up to `queries` queries and `keys` keys each."""
    return {"name": name, "op": op, "seqs": seqs, "queries": queries, "keys": keys, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "mix": mix}


def listed():
    return [
        # a server's step: 64 users' new tokens into their pages
        _cached("append decode", "append", 64, 1, 510, 32, 8, 128, 16, 16, "bf16", 1),
        # the next pieces of four prompts, kept in 16 bits, with what came before read back for attention
        _cached("piece 16 bits", "piece", 4, 2048, 4099, 32, 8, 128, 16, 64, "bf16", 2),
        # one long prompt's piece into a cache of 4 bits
        _cached("piece 4 bits", "piece", 1, 4096, 20001, 32, 8, 128, 4, 64, "bf16", 3),
        # one user's next token: latency, and a long axis with one row of queries per head
        _cached("cached one", "cached", 1, 1, 1801, 32, 8, 128, 16, 16, "bf16", 4),
        # a server's step: 64 users, caches of very different lengths
        _cached("cached batch", "cached", 64, 1, 8191, 32, 8, 128, 16, 64, "bf16", 5),
        # drafted tokens checked together: up to five new tokens for each user, small heads
        _cached("cached drafts", "cached", 24, 5, 4099, 16, 4, 64, 16, 32, "fp16", 6),
        # one user far into a long document, in 4 bits
        _cached("cached long 4 bits", "cached", 1, 1, 131071, 64, 8, 128, 4, 64, "bf16", 7),
        # many users on the memory that 4 bits free
        _cached("cached batch 4 bits", "cached", 128, 1, 16383, 32, 8, 128, 4, 64, "bf16", 8),
        # a video's tokens in front of attention: positions in time, height and width
        _rope("rope video", "rope", 16411, 32, 8, 128, 128, 3, False, "bf16"),
        # the gradient of that in a training step, positions of an image's rows and columns
        _rope("rope gradient", "rope_grad", 8192, 16, 16, 80, 80, 2, True, "bf16"),
        # a decoder's next tokens against an encoder's states
        _cross("cross decode", "cross", 48, 1, 1500, 20, 20, 64, "fp16", 9),
        # a training step of an encoder-decoder's cross attention
        _cross("cross train", "cross_train", 8, 1030, 2050, 16, 4, 128, "bf16", 10),
    ]


def draw(rng):
    def log(lo, hi):
        return min(hi, int(lo * math.exp(rng.random() * math.log((hi + 1) / lo))))

    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 4, 5, 8])
    dim = rng.choice([64, 80, 96, 128])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    op = rng.choice(["append", "piece", "cached", "cached", "cached", "rope", "rope_grad", "cross", "cross_train"])
    mix = rng.randrange(1 << 20)
    if op.startswith("rope"):
        c = _rope("", op, log(1, 16384), heads, kv_heads, dim, rng.choice([dim, dim, dim // 2]), rng.choice([1, 2, 3, 4]), rng.random() < 0.4, rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    elif op.startswith("cross"):
        c = _cross("", op, log(1, 48), 1 if op == "cross" and rng.random() < 0.4 else log(1, 2048), log(1, 2048), min(heads, 20), min(heads, 20), dim, dtype, mix)
        if heads <= 20:
            c["kv_heads"] = kv_heads
        while c["seqs"] * c["heads"] * c["queries"] * c["keys"] > 1 << 29:  # the plain form's scores
            c["seqs"] = max(1, c["seqs"] // 2)
            c["queries"] = max(1, c["queries"] // 2)
    else:
        bits = 16 if op == "append" else rng.choice([16, 4])
        dim = rng.choice([64, 96, 128]) if bits == 4 else dim
        seqs = log(1, 128)
        new = 1 if op == "append" and rng.random() < 0.5 else log(1, 2048) if op != "cached" else rng.choice([1, 1, 1, 2, 3, 5, 8])
        c = _cached("", op, seqs, new, log(1, 16383), heads, kv_heads, dim, bits, rng.choice([16, 32, 64, 128]), dtype, mix)
        most = (1 << 31 if bits == 4 else 1 << 29) if op == "cached" else 1 << 26
        while c["seqs"] * (c["longest"] + c["new"]) * kv_heads * dim > most or c["seqs"] * c["new"] > 16384:  # the plain form's padded keys
            c["seqs"] = max(1, c["seqs"] // 2)
            c["longest"] = max(1, c["longest"] // 2) if c["seqs"] == 1 else c["longest"]
            c["new"] = c["new"] if op == "cached" else max(1, c["new"] // 2)
    del c["name"]
    return c


def lengths(case):
    """(new tokens or queries, keys with the new ones) of every sequence."""
    r = random.Random(case["mix"])
    n = case["seqs"]
    if case["op"].startswith("cross"):
        q = [case["queries"]] + [r.randint(1 + case["queries"] * 3 // 4, case["queries"]) if case["queries"] > 1 else 1 for _ in range(n - 1)]
        return q, [case["keys"]] + [max(1, int(case["keys"] * (0.5 + 0.5 * r.random()))) for _ in range(n - 1)]
    q = [case["new"]] + [r.randint(max(1, case["new"] // 2), case["new"]) for _ in range(n - 1)]
    # spread over the logarithm: a few long caches, many short ones
    before = [case["longest"]] + [int(math.exp(r.random() * math.log(case["longest"] + 1))) for _ in range(n - 1)]
    return q, [x + y for x, y in zip(q, before)]


def _tables(columns, positions, base=10000.0):
    rate = base ** (-torch.arange(columns, device="cuda", dtype=torch.float64) / max(columns, 1))
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * rate
    return angle.cos().float(), angle.sin().float()


def _pair_axes(pairs, axes):
    """The axis that turns each pair: sections of about the same number, the first one smaller."""
    first = max(1, pairs // axes * 3 // 4)
    return [0] * pairs if axes == 1 else [0 if j < first else 1 + (j - first) * (axes - 1) // (pairs - first) for j in range(pairs)]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, dtype, heads, kv, dim = case["op"], DTYPES[case["dtype"]], case["heads"], case["kv_heads"], case["dim"]

    def normal(*shape, std=1.0, to=dtype):
        return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(to)

    s = {"case": case}
    if op.startswith("rope"):
        n, half = case["total"], case["rotated"] // 2
        fused = normal(n, heads + 2 * kv, dim)  # the projection's output: queries, keys, values
        s["q"], s["k"] = fused[:, :heads], fused[:, heads:heads + kv]
        s["positions"] = torch.randint(0, POSITIONS, (case["axes"], n), generator=g, device="cuda", dtype=torch.int32)
        s["axes"] = _pair_axes(half, case["axes"])
        s["cos"], s["sin"] = _tables(half, POSITIONS)
        return s
    q_len, k_len = lengths(case)
    n = len(q_len)

    def whole(x):
        return torch.tensor(x, device="cuda", dtype=torch.int32)
    if op.startswith("cross"):
        s["q"], s["k"] = normal(sum(q_len), heads, dim, std=1.5), normal(sum(k_len), kv, dim)
        s["v"] = normal(sum(k_len), 2 * kv, dim)[:, kv:]  # where the projection left it
        if op == "cross_train":
            s["do"] = normal(sum(q_len), heads, dim)
        if own:
            import paper_2608_13757_gb300 as sg
            s["plan"] = sg.sync_attn_plan(q_len, k_len, heads, kv, dim, dtype, train=op == "cross_train", causal=False)
        else:
            s["q_at"], s["q_ok"] = _padded(q_len)
            s["k_at"], s["k_ok"] = _padded(k_len)
        return s
    page, bits = case["page"], case["bits"]
    of = [-(-x // page) for x in k_len]
    width, used = max(of), sum(of)
    pages = used + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)  # as they lie after long service
    table = torch.full((n, width), -1, device="cuda", dtype=torch.int32)
    table[torch.arange(width, device="cuda") < whole(of)[:, None]] = order[:used]
    s["table"], s["lens"] = table, whole(k_len)
    s["starts"] = None if case["new"] == 1 else whole([sum(q_len[:i]) for i in range(n + 1)])
    if bits == 16:
        s["cache"] = {"k": normal(pages, kv, page, dim), "v": normal(pages, kv, page, dim)}
    else:
        s["cache"] = {}
        for x in ("k", "v"):
            a, b = (normal(pages, kv, page, dim // 2, std=3.0, to=torch.float32).round_().clamp_(-7, 7).add_(8).to(torch.uint8) for _ in range(2))
            s["cache"][x] = a | b << 4
            s["cache"][x + "_scale"] = (0.3 * torch.exp(normal(pages, kv, page, dim // 32, std=0.3, to=torch.float32))).half()
    if op == "cached":
        s["q"] = normal(sum(q_len), heads, dim, std=1.5)
        s["longest"] = max(q_len)
    else:
        fused = normal(sum(q_len), heads + 2 * kv, dim)
        s["q"], s["k"], s["v"] = fused[:, :heads], fused[:, heads:heads + kv], fused[:, heads + kv:]
        s["cos"], s["sin"] = _tables(dim // 2, max(k_len))
        if op == "piece":
            s["read_starts"], s["read_rows"] = whole([sum(k_len[:i]) for i in range(n + 1)]), sum(k_len)
    if own:
        import paper_2608_13757_gb300 as sg
        s["handle"] = sg.sync_kv_cache(pages, page, kv, dim, dtype, bits=bits)
        for x, t in s["cache"].items():
            getattr(s["handle"], x).copy_(t)
            s["cache"][x] = getattr(s["handle"], x)
        return s
    s["q_at"], s["q_ok"] = _padded(q_len)
    s["seen"] = s["lens"].long()[:, None] - whole(q_len)[:, None] + torch.arange(max(q_len), device="cuda") + 1  # keys that a new token sees
    at = torch.repeat_interleave(torch.arange(n, device="cuda"), whole(q_len).long())
    s["pos"] = (s["seen"] - 1)[s["q_ok"]]
    s["to"] = table.long()[at, s["pos"] // page], s["pos"] % page
    if op == "piece":
        at = torch.repeat_interleave(torch.arange(n, device="cuda"), s["lens"].long())
        pos = torch.arange(sum(k_len), device="cuda") - s["read_starts"].long()[at]
        s["from"] = table.long()[at, pos // page], pos % page
    return s


def _padded(lens):
    """[sequence, token] row numbers of packed rows, and which of them are tokens."""
    n = torch.tensor(lens, device="cuda")
    i = torch.arange(max(lens), device="cuda")
    return ((n.cumsum(0) - n)[:, None] + i).clamp(max=sum(lens) - 1), i < n[:, None]


def run(s):
    c = s["case"]
    op = c["op"]
    if own:
        import paper_2608_13757_gb300 as sg
        if op == "rope":
            return sg.sync_rope(s["q"], s["k"], s["cos"], s["sin"], s["positions"], axes=s["axes"], interleaved=c["interleaved"])
        if op == "rope_grad":
            return sg.sync_rope_backward(s["q"], s["k"], s["cos"], s["sin"], s["positions"], axes=s["axes"], interleaved=c["interleaved"])
        if op == "cross":
            return sg.sync_attn_forward(s["plan"], s["q"], s["k"], s["v"])
        if op == "cross_train":
            o, lse = sg.sync_attn_forward(s["plan"], s["q"], s["k"], s["v"], lse=True)
            return (o,) + tuple(sg.sync_attn_backward(s["plan"], s["q"], s["k"], s["v"], o, lse, s["do"]))
        if op == "cached":
            return sg.sync_cache_attn(s["handle"], s["q"], s["table"], s["lens"], s["starts"], max_new=s["longest"])
        q = sg.sync_cache_append(s["handle"], s["k"], s["v"], s["table"], s["lens"], s["starts"], q=s["q"], cos=s["cos"], sin=s["sin"])
        if op == "piece":
            return (q,) + tuple(sg.sync_cache_read(s["handle"], s["table"], s["lens"], s["read_starts"], s["read_rows"]))
        return q, s["cache"]
    if op.startswith("rope"):
        axis = torch.tensor(s["axes"], device="cuda")
        at = s["positions"].long()[axis].T, torch.arange(len(s["axes"]), device="cuda")
        cos, sin = s["cos"][at][:, None], s["sin"][at][:, None]
        sin = -sin if op == "rope_grad" else sin
        return tuple(_turn(x.float(), cos, sin, c["interleaved"]).to(x.dtype) for x in (s["q"], s["k"]))
    if op.startswith("cross"):
        return _plain_cross(s)
    if op == "cached":
        return _plain_cached(s)
    cos, sin = s["cos"][s["pos"]][:, None], s["sin"][s["pos"]][:, None]
    q, k = (_turn(s[x].float(), cos, sin, False) for x in "qk")
    q = q.to(s["q"].dtype)
    (p, i), h = s["to"], torch.arange(c["kv_heads"], device="cuda")
    at = p[:, None], h, i[:, None]
    for x, t in (("k", k), ("v", s["v"].float())):
        if c["bits"] == 16:
            s["cache"][x][at] = t.to(s["v"].dtype)
        else:
            s["cache"][x][at], s["cache"][x + "_scale"][at] = _pack(t)
    if op == "append":
        return q, s["cache"]
    p, i = s["from"]
    at = p[:, None], h, i[:, None]
    if c["bits"] == 16:
        return q, s["cache"]["k"][at], s["cache"]["v"][at]
    return (q,) + tuple(_unpack(s["cache"][x][at], s["cache"][x + "_scale"][at]).to(q.dtype) for x in "kv")


def _turn(x, cos, sin, interleaved):
    """The rotation of each pair of a head's first entries."""
    n = 2 * cos.shape[-1]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:n:2], x[..., 1:n:2]
        y[..., 0:n:2], y[..., 1:n:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :n // 2], x[..., n // 2:n]
        y[..., :n // 2], y[..., n // 2:n] = a * cos - b * sin, b * cos + a * sin
    return y


def _pack(x):
    """Codes and scales of rows."""
    g = x.shape[-1] // 32
    x = x.unflatten(-1, (g, 4, 8))
    scale = (x.abs().amax((-2, -1)) / torch.full((), 7.0, device=x.device)).half()
    by = scale.float()[..., None, None]
    code = (torch.where(by > 0, x / by, 0.0).round().clamp(-7, 7) + 8).to(torch.uint8).transpose(-3, -2)
    return (code[..., 0::2] | code[..., 1::2] << 4).flatten(-3), scale


def _unpack(codes, scale):
    """The values that rows of codes and scales stand for."""
    x = codes.unflatten(-1, (4, scale.shape[-1], 4))
    x = torch.stack((x & 15, x >> 4), -1).flatten(-2).transpose(-3, -2)
    return ((x.float() - 8) * scale.float()[..., None, None]).flatten(-3)


def _plain_cached(s):
    c, q = s["case"], s["q"]
    n, m = s["q_at"].shape
    kv, g, d = c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"]
    table = s["table"].long().clamp(min=0)

    def keys(x):  # [sequences * key heads, keys, dim]
        t = s["cache"][x][table]
        t = t.float() if c["bits"] == 16 else _unpack(t, s["cache"][x + "_scale"][table])
        return t.transpose(1, 2).reshape(n * kv, -1, d)
    qf = q[s["q_at"]].float().view(n, m, kv, g, d).permute(0, 2, 3, 1, 4).reshape(n * kv, g * m, d)
    p = torch.bmm(qf, keys("k").transpose(1, 2)).mul_(d ** -0.5)
    hidden = torch.arange(p.shape[-1], device="cuda") >= s["seen"][..., None]
    p.view(n, kv, g, m, -1).masked_fill_(hidden[:, None, None], -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True)).exp_()
    o = torch.bmm(p.div_(p.sum(-1, keepdim=True)), keys("v"))
    o = o.view(n, kv, g, m, d).permute(0, 3, 1, 2, 4).reshape(n, m, kv * g, d)
    return o[s["q_ok"]].to(q.dtype)


def _plain_cross(s):
    c, q, k, v = s["case"], s["q"], s["k"], s["v"]
    (n, lq), lk = s["q_at"].shape, s["k_at"].shape[1]
    kv, g, d = c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"]

    def rows(x):  # [sequences * key heads, heads of the group * queries, dim]
        return x[s["q_at"]].float().view(n, lq, kv, g, d).permute(0, 2, 3, 1, 4).reshape(n * kv, g * lq, d)

    def keys(x):
        return x[s["k_at"]].float().permute(0, 2, 1, 3).reshape(n * kv, lk, d)

    def rows_back(x):
        return x.view(n, kv, g, lq, d).permute(0, 3, 1, 2, 4).reshape(n, lq, kv * g, d)[s["q_ok"]].to(q.dtype)

    def keys_back(x):
        return x.view(n, kv, lk, d).permute(0, 2, 1, 3)[s["k_ok"]].to(k.dtype)

    qf, kf, vf = rows(q), keys(k), keys(v)
    scale = d ** -0.5
    p = torch.bmm(qf, kf.transpose(1, 2)).mul_(scale)
    p.view(n, kv, g * lq, lk).masked_fill_(~s["k_ok"][:, None, None], -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True)).exp_()
    p = p.div_(p.sum(-1, keepdim=True))
    o = torch.bmm(p, vf)
    if c["op"] == "cross":
        return rows_back(o)
    # rows past a shorter sequence's end hold another sequence's queries: no gradient comes from them
    do = rows(s["do"]) * s["q_ok"][:, None, None, :, None].expand(n, kv, g, lq, 1).reshape(n * kv, g * lq, 1)
    dv = torch.bmm(p.transpose(1, 2), do)
    ds = torch.bmm(do, vf.transpose(1, 2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    return rows_back(o), rows_back(torch.bmm(ds, kf)), keys_back(torch.bmm(ds.transpose(1, 2), qf)), keys_back(dv)


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    heads, kv, dim = case["heads"], case["kv_heads"], case["dim"]
    if case["op"].startswith("rope"):
        n, row = case["total"], (heads + kv) * dim
        angles = min(n, POSITIONS) * case["rotated"] * 4
        return {"bytes": 2 * n * row * size + angles + 4 * n * case["axes"], "flops": 3 * n * row}
    q, k = lengths(case)
    a, b = sum(q) * heads * dim * size, sum(k) * kv * dim * size
    if case["op"] == "cross_train":
        # q, k, v, do read, o, dq, dk, dv written; two products forward and five backward
        return {"bytes": 4 * a + 4 * b, "flops": 14 * dim * heads * sum(x * y for x, y in zip(q, k))}
    if case["op"] == "cross":
        return {"bytes": 2 * a + 2 * b, "flops": 4 * dim * heads * sum(x * y for x, y in zip(q, k))}
    row = kv * (dim * 2 if case["bits"] == 16 else dim // 2 + dim // 32 * 2)  # bytes of a token's keys in the cache
    if case["op"] == "cached":
        pairs = sum(x * y - x * (x - 1) // 2 for x, y in zip(q, k))
        return {"bytes": 2 * a + 2 * sum(k) * row, "flops": 4 * dim * heads * pairs}
    new = 2 * a + 2 * sum(q) * (kv * dim * size + row) + sum(q) * dim * 4
    if case["op"] == "append":
        return {"bytes": new, "flops": 3 * sum(q) * (heads + kv) * dim}
    return {"bytes": new + 2 * sum(k) * (kv * dim * size + row), "flops": 3 * sum(q) * (heads + kv) * dim}


def exact(case, seed):
    """The definitions in 64 bits, one sequence at a time."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    heads, g, dim, op = case["heads"], case["heads"] // case["kv_heads"], case["dim"], case["op"]
    if op.startswith("rope"):
        return _exact_rope(case, s)
    q_len, k_len = lengths(case)
    a, b = 0, 0
    if op.startswith("cross"):
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        grads = [torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (s["q"], s["k"], s["v"])]
        for n, m in zip(q_len, k_len):
            for h in range(heads):
                q, k, v = s["q"][a:a + n, h].double(), s["k"][b:b + m, h // g].double(), s["v"][b:b + m, h // g].double()
                w = torch.softmax(q @ k.T / math.sqrt(dim), 1)
                out[a:a + n, h] = w @ v
                if op == "cross_train":
                    go = s["do"][a:a + n, h].double()
                    grads[2][b:b + m, h // g] += w.T @ go
                    gw = go @ v.T
                    ge = w * (gw - (gw * w).sum(1, keepdim=True)) / math.sqrt(dim)
                    grads[0][a:a + n, h] = ge @ k
                    grads[1][b:b + m, h // g] += ge.T @ q
            a, b = a + n, b + m
        return (out, *grads) if op == "cross_train" else out
    page, bits = case["page"], case["bits"]
    cache = {x: t.double() for x, t in s["cache"].items()} if bits == 16 else s["cache"]
    # where each entry of a row of 4-bit codes is
    d = torch.arange(dim, device="cuda")
    byte, shift = 4 * (dim // 32 * (d // 8 % 4) + d // 32) + d % 8 // 2, 4 * (d % 2)

    def values(x, rows, where):  # of `rows` tokens from cache[x]
        t = cache[x][where]
        if bits == 4:
            t = ((t[..., byte].int() >> shift & 15) - 8) * cache[x + "_scale"][where].double()[..., d // 32]
        return t[:rows]
    if op == "cached":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for i, (n, m) in enumerate(zip(q_len, k_len)):
            used = s["table"][i, :-(-m // page)].long()
            seen = torch.ones(n, m, dtype=torch.bool, device="cuda").tril(m - n)
            for h in range(case["kv_heads"]):
                k, v = (values(x, None, (used, h)).reshape(-1, dim)[:m] for x in "kv")
                q = s["q"][a:a + n, h * g:(h + 1) * g].double()
                e = torch.einsum("nhd,kd->hnk", q, k) / math.sqrt(dim)
                out[a:a + n, h * g:(h + 1) * g] = torch.einsum("hnk,kd->nhd", torch.softmax(e.masked_fill(~seen, -math.inf), 2), v)
            a += n
        return out
    turn = torch.complex(s["cos"].double(), s["sin"].double())[s["pos"]][:, None]

    def turned(x):
        z = torch.complex(x[..., :dim // 2].double(), x[..., dim // 2:].double()) * turn
        return torch.cat((z.real, z.imag), -1)
    q, rows = turned(s["q"]), {"k": turned(s["k"]), "v": s["v"].double()}
    if bits == 4:  # the values that the codes will stand for
        for x, t in rows.items():
            t = t.unflatten(-1, (-1, 32))
            by = (t.abs().amax(-1, keepdim=True) / 7).half().double()
            rows[x] = torch.where(by > 0, torch.clamp(torch.round(t / by), -7, 7) * by, 0.0).flatten(-2)
    if op == "append":
        for x, t in rows.items():
            cache[x][s["to"][0], :, s["to"][1]] = t
        return q, cache
    res = []
    for x, t in rows.items():
        y, a, b = [], 0, 0
        for i, (n, m) in enumerate(zip(q_len, k_len)):
            used = s["table"][i, :-(-m // page)].long()
            old = values(x, None, (used,)).transpose(1, 2).flatten(0, 1)[:m - n]
            y += [old, t[a:a + n]]
            a += n
        res.append(torch.cat(y))
    return q, *res


def _exact_rope(case, s):
    n, r = case["total"], case["rotated"]
    way = -1.0 if case["op"] == "rope_grad" else 1.0
    cos, sin = (torch.stack([t[s["positions"][a].long(), j].double() for j, a in enumerate(s["axes"])], 1)[:, None] for t in (s["cos"], way * s["sin"]))
    one = torch.arange(0, r, 2, device="cuda") if case["interleaved"] else torch.arange(r // 2, device="cuda")
    two = one + (1 if case["interleaved"] else r // 2)
    res = []
    for x in (s["q"], s["k"]):
        x = x.double()
        y = x.clone()
        y[:, :, one] = x[:, :, one] * cos - x[:, :, two] * sin
        y[:, :, two] = x[:, :, two] * cos + x[:, :, one] * sin
        res.append(y)
    return tuple(res)
