"""The measured operators: attention over packed sequences and the pass in front of it.

Two operators, each with its gradient:

  attention   causal attention with grouped heads over sequences of different
              lengths packed into one tensor: a whole prompt, a training step
              (forward and backward), and one new token per sequence against
              the keys and values kept so far
  norm-rope   root-mean-square norm of the query and key heads with the
              position rotation in the same pass, and its gradient

A case holds plain sizes; the sequences' lengths follow from them
(`lengths`), so the work of a case does not depend on the seed.  `run` makes
one pass: with `own` false in elementary torch operations in 32 bits, with
`own` true through the package.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


def _attention(name, op, seqs, total, prefix, heads, kv_heads, dim, dtype, mix):
    """seqs sequences, total query tokens, up to `prefix` earlier keys each;
    `mix` picks the split of the totals into sequences."""
    return {"name": name, "op": op, "seqs": seqs, "total": total, "prefix": prefix, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "mix": mix}


def _norm(name, op, total, heads, kv_heads, dim, rotated, interleaved, dtype):
    return {"name": name, "op": op, "total": total, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rotated": rotated, "interleaved": interleaved, "dtype": dtype}


def listed():
    return [
        # one user's next token: latency, and a long axis with one row of queries per head
        _attention("decode one", "decode", 1, 1, 1801, 32, 8, 128, "bf16", 1),
        # a server's step: 64 users, one token each, caches of very different lengths
        _attention("decode batch", "decode", 64, 64, 8191, 32, 8, 128, "bf16", 2),
        # a few short prompts of an interactive service, small heads, odd lengths
        _attention("short prompts", "prompt", 13, 901, 0, 16, 4, 64, "fp16", 3),
        # a service's prompt batch: ragged prompts packed together
        _attention("packed prompts", "prompt", 11, 12289, 0, 32, 8, 128, "bf16", 4),
        # the next pieces of prompts whose beginnings are already in the cache
        _attention("prompt pieces", "prompt", 5, 1535, 4099, 32, 4, 128, "bf16", 5),
        # one long prompt, a key head for every query head
        _attention("long prompt", "prompt", 1, 8192, 0, 32, 32, 128, "bf16", 6),
        # fine-tuning a small model on short packed documents
        _attention("train short", "train", 9, 2003, 0, 12, 4, 64, "fp16", 7),
        # a training step over packed documents
        _attention("train packed", "train", 7, 8192, 0, 32, 8, 128, "bf16", 8),
        # a training step over one long document
        _attention("train long", "train", 1, 8192, 0, 32, 32, 128, "bf16", 9),
        # the pass in front of a server's decode step
        _norm("norm decode", "norm", 64, 32, 8, 128, 128, False, "bf16"),
        # the pass in front of a prompt batch
        _norm("norm prompts", "norm", 16411, 32, 8, 128, 128, False, "bf16"),
        # its gradient in a training step
        _norm("norm gradient", "norm_grad", 8192, 32, 8, 128, 128, False, "bf16"),
    ]


def draw(rng):
    def log(lo, hi):
        return min(hi, int(lo * math.exp(rng.random() * math.log((hi + 1) / lo))))

    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 5, 8])
    heads = heads if heads <= 20 else kv_heads * max(1, 16 // kv_heads)
    dim = rng.choice([64, 80, 96, 128])
    if 24 * 128 in (dim * heads, dim * (heads + kv_heads), dim * (heads + 2 * kv_heads)):
        dim = 80
    op = rng.choice(["decode", "prompt", "prompt", "train", "train", "norm", "norm_grad"])
    if op.startswith("norm"):
        rotated = rng.choice([dim, dim, dim // 2])
        c = _norm("", op, log(1, 16384), heads, kv_heads, dim, rotated, rng.random() < 0.3, rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    elif op == "decode":
        seqs = log(1, 64)
        c = _attention("", op, seqs, seqs, log(1, 8191), heads, kv_heads, dim, rng.choice(["bf16", "fp16"]), rng.randrange(1 << 20))
    else:
        seqs = log(1, 32)
        prefix = log(1, 4096) if op == "prompt" and rng.random() < 0.4 else 0
        c = _attention("", op, seqs, log(seqs, 8192), prefix, heads, kv_heads, dim, rng.choice(["bf16", "fp16"]), rng.randrange(1 << 20))
        while _scores(c) > 1 << 31:  # the plain form's scores, padded to the longest sequence
            c["total"] = max(seqs, c["total"] // 2)
            c["prefix"] //= 2
    del c["name"]
    return c


def lengths(case):
    """(query tokens, keys) of every sequence."""
    r = random.Random(case["mix"])
    n = case["seqs"]
    if case["op"] == "decode":
        q = [1] * n
    else:
        weight = [0.15 + r.random() for _ in range(n)]
        q = [max(1, int(case["total"] * w / sum(weight))) for w in weight]
        q[q.index(max(q))] += case["total"] - sum(q)
        q = [max(1, x) for x in q]
    most = case["prefix"]
    if case["op"] == "decode":  # spread over the logarithm: a few long caches, many short ones
        before = [most if n == 1 else int(math.exp(r.random() * math.log(most + 1))) for _ in range(n)]
    else:
        before = [r.randint(0, most) for _ in range(n)]
    return q, [x + y for x, y in zip(q, before)]


def _scores(case):
    q, k = lengths(case)
    return len(q) * case["heads"] * max(q) * max(k)


def _starts(case):
    """First row of every sequence in the query and in the key tensors.  Prompts
    are packed; a decode step's caches have room for the longest."""
    q, k = lengths(case)
    room = [max(k)] * len(k) if case["op"] == "decode" else k
    return [sum(q[:b]) for b in range(len(q))], [sum(room[:b]) for b in range(len(k))], sum(q), sum(room)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype, heads, kv_heads, dim = DTYPES[case["dtype"]], case["heads"], case["kv_heads"], case["dim"]

    def normal(*shape, std=1.0, to=dtype):
        return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(to)

    s = {"case": case}
    if case["op"] in ("norm", "norm_grad"):
        n, half = case["total"], case["rotated"] // 2
        fused = normal(n, heads + 2 * kv_heads, dim, std=1.7)  # the projection's output: queries, keys, values
        s["q"], s["k"] = fused[:, :heads], fused[:, heads:heads + kv_heads]
        s["wq"], s["wk"] = 1 + normal(dim, std=0.1, to=torch.float32), 1 + normal(dim, std=0.1, to=torch.float32)
        s["wq"], s["wk"] = s["wq"].to(dtype), s["wk"].to(dtype)
        s["positions"] = torch.randint(0, 8192, (n,), generator=g, device="cuda", dtype=torch.int32)
        rate = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        angle = torch.arange(8192, device="cuda", dtype=torch.float64)[:, None] * rate
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        if case["op"] == "norm_grad":
            s["dq"], s["dk"] = normal(n, heads, dim), normal(n, kv_heads, dim)
        return s
    q_len, k_len = lengths(case)
    q_start, k_start, q_rows, k_rows = _starts(case)
    s["q"], s["k"] = normal(q_rows, heads, dim, std=1.5), normal(k_rows, kv_heads, dim)
    if case["op"] == "train":
        s["v"] = normal(k_rows, heads + 2 * kv_heads, dim)[:, heads + kv_heads:]  # where the projection left it
        s["do"] = normal(q_rows, heads, dim)
    else:
        s["v"] = normal(k_rows, kv_heads, dim)
    if own:
        import paper_2608_13757_gb300 as sg
        s["plan"] = sg.sync_attn_plan(q_len, k_len, heads, kv_heads, dim, dtype, q_starts=q_start, k_starts=k_start, train=case["op"] == "train")
    else:
        lq, lk, aq, ak = (torch.tensor(x, device="cuda") for x in (q_len, k_len, q_start, k_start))
        i, j = torch.arange(max(q_len), device="cuda"), torch.arange(max(k_len), device="cuda")
        s["q_ok"], s["k_ok"] = i < lq[:, None], j < lk[:, None]
        s["q_at"], s["k_at"] = (aq[:, None] + i).clamp(max=q_rows - 1), (ak[:, None] + j).clamp(max=k_rows - 1)
        s["last"] = i + (lk - lq)[:, None]  # the last key that a query sees
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        import paper_2608_13757_gb300 as sg
        interleaved = bool(s["case"].get("interleaved"))
        if op == "norm":
            return sg.sync_qk_norm_rope(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["positions"], eps=EPS, interleaved=interleaved)
        if op == "norm_grad":
            return sg.sync_qk_norm_rope_backward(s["q"], s["k"], s["dq"], s["dk"], s["wq"], s["wk"], s["cos"], s["sin"], s["positions"], eps=EPS, interleaved=interleaved)
        if op == "train":
            o, lse = sg.sync_attn_forward(s["plan"], s["q"], s["k"], s["v"], lse=True)
            return (o,) + tuple(sg.sync_attn_backward(s["plan"], s["q"], s["k"], s["v"], o, lse, s["do"]))
        return sg.sync_attn_forward(s["plan"], s["q"], s["k"], s["v"])
    if op == "norm":
        return _plain_norm(s, s["q"], s["wq"]), _plain_norm(s, s["k"], s["wk"])
    if op == "norm_grad":
        dq, dwq = _plain_norm_grad(s, s["q"], s["wq"], s["dq"])
        dk, dwk = _plain_norm_grad(s, s["k"], s["wk"], s["dk"])
        return dq, dk, dwq, dwk
    return _plain_attention(s)


def _rotate(s, x, sign):
    """The rotation of each pair of a head's first entries by its position's angles."""
    c = s["case"]
    n = c["rotated"]
    cos, sin = s["cos"][s["positions"].long()][:, None], sign * s["sin"][s["positions"].long()][:, None]
    y = x.clone()
    if c["interleaved"]:
        a, b = x[..., 0:n:2], x[..., 1:n:2]
        y[..., 0:n:2], y[..., 1:n:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :n // 2], x[..., n // 2:n]
        y[..., :n // 2], y[..., n // 2:n] = a * cos - b * sin, b * cos + a * sin
    return y


def _plain_norm(s, x, w):
    f = x.float()
    f = f * torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS) * w.float()
    return _rotate(s, f, 1.0).to(x.dtype)


def _plain_norm_grad(s, x, w, dy):
    f = x.float()
    r = torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS)
    f = f * r
    d = _rotate(s, dy.float(), -1.0)
    dw = (d * f).sum((0, 1))
    d = d * w.float()
    return (r * (d - f * (d * f).mean(-1, keepdim=True))).to(x.dtype), dw.to(w.dtype)


def _plain_attention(s):
    c, q, k, v = s["case"], s["q"], s["k"], s["v"]
    n, lq, lk = s["q_at"].shape[0], s["q_at"].shape[1], s["k_at"].shape[1]
    hk, g, d = c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"]

    def rows(x):  # [sequences * key heads, heads of the group * queries, dim]
        return x[s["q_at"]].float().view(n, lq, hk, g, d).permute(0, 2, 3, 1, 4).reshape(n * hk, g * lq, d)

    def keys(x):
        return x[s["k_at"]].float().permute(0, 2, 1, 3).reshape(n * hk, lk, d)

    def rows_back(x):
        y = torch.zeros_like(q)
        x = x.view(n, hk, g, lq, d).permute(0, 3, 1, 2, 4).reshape(n, lq, hk * g, d)
        y[s["q_at"][s["q_ok"]]] = x[s["q_ok"]].to(q.dtype)
        return y

    def keys_back(x):
        y = torch.zeros_like(k)
        y[s["k_at"][s["k_ok"]]] = x.view(n, hk, lk, d).permute(0, 2, 1, 3)[s["k_ok"]].to(k.dtype)
        return y

    qf, kf, vf = rows(q), keys(k), keys(v)
    scale = d ** -0.5
    p = torch.bmm(qf, kf.transpose(1, 2)).mul_(scale)
    hidden = torch.arange(lk, device=q.device) > s["last"][..., None]
    hidden = (hidden | ~s["k_ok"][:, None]).view(n, 1, 1, lq, lk)
    p.view(n, hk, g, lq, lk).masked_fill_(hidden, -math.inf)
    m = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    l = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(l == 0, 1.0, l))
    o = torch.bmm(p, vf)
    if c["op"] != "train":
        return rows_back(o)
    # rows past a shorter sequence's end hold another sequence's queries: no gradient comes from them
    do = rows(s["do"]) * s["q_ok"][:, None, None, :, None].expand(n, hk, g, lq, 1).reshape(n * hk, g * lq, 1)
    dv = torch.bmm(p.transpose(1, 2), do)
    ds = torch.bmm(do, vf.transpose(1, 2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    return rows_back(o), rows_back(torch.bmm(ds, kf)), keys_back(torch.bmm(ds.transpose(1, 2), qf)), keys_back(dv)


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] in ("norm", "norm_grad"):
        n, row = case["total"], (case["heads"] + case["kv_heads"]) * case["dim"]
        grad = case["op"] == "norm_grad"
        angles = min(n, 8192) * case["rotated"] * 4
        return {"bytes": (3 if grad else 2) * n * row * size + angles + 4 * n + (4 if grad else 2) * case["dim"] * size, "flops": (16 if grad else 8) * n * row}
    q, k = lengths(case)
    pairs = sum(sum(y - x + 1 + i for i in range(x)) for x, y in zip(q, k)) * case["heads"]
    a, b = sum(q) * case["heads"] * case["dim"] * size, sum(k) * case["kv_heads"] * case["dim"] * size
    if case["op"] == "train":
        # q, k, v, do read, o, dq, dk, dv written; two products forward and five backward
        return {"bytes": 4 * a + 4 * b, "flops": 14 * case["dim"] * pairs}
    return {"bytes": 2 * a + 2 * b, "flops": 4 * case["dim"] * pairs}


def exact(case, seed):
    """The definitions in 64 bits, one sequence and one head at a time."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] in ("norm", "norm_grad"):
        return _exact_norm(case, s)
    heads, g, dim = case["heads"], case["heads"] // case["kv_heads"], case["dim"]
    q_len, k_len = lengths(case)
    q_start, k_start, _, _ = _starts(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    train = case["op"] == "train"
    grads = [torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (s["q"], s["k"], s["v"])] if train else []
    for a, n, b, m in zip(q_start, q_len, k_start, k_len):
        seen = torch.ones(n, m, dtype=torch.bool, device="cuda").tril(m - n)
        for h in range(heads):
            q, k, v = s["q"][a:a + n, h].double(), s["k"][b:b + m, h // g].double(), s["v"][b:b + m, h // g].double()
            e = torch.where(seen, q @ k.T / math.sqrt(dim), torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
            w = torch.softmax(e, 1)
            o = w @ v
            out[a:a + n, h] = o
            if train:
                go = s["do"][a:a + n, h].double()
                grads[2][b:b + m, h // g] += w.T @ go
                gw = go @ v.T
                ge = w * (gw - (gw * w).sum(1, keepdim=True)) / math.sqrt(dim)
                grads[0][a:a + n, h] = ge @ k
                grads[1][b:b + m, h // g] += ge.T @ q
    return (out, *grads) if train else out


def _exact_norm(case, s):
    n, r, dim = case["total"], case["rotated"], case["dim"]
    at = s["positions"].long()
    cos, sin = s["cos"].double()[at], s["sin"].double()[at]
    turn = torch.zeros(n, dim, dim, dtype=torch.float64, device="cuda") if n * dim * dim <= 1 << 26 else None
    one, two = (range(0, r, 2), range(1, r, 2)) if case["interleaved"] else (range(r // 2), range(r // 2, r))
    one, two = torch.tensor(list(one), device="cuda"), torch.tensor(list(two), device="cuda")

    def rotated(x, way):  # as a matrix for each token where that fits, by its pairs where it does not
        if turn is not None:
            turn.zero_()
            turn[:, torch.arange(dim), torch.arange(dim)] = 1.0
            turn[:, one, one] = cos
            turn[:, two, two] = cos
            turn[:, one, two] = -way * sin
            turn[:, two, one] = way * sin
            return torch.einsum("nij,nhj->nhi", turn, x)
        u, w, y = x[:, :, one], x[:, :, two], x.clone()
        y[:, :, one] = u * cos[:, None] - w * sin[:, None] * way
        y[:, :, two] = w * cos[:, None] + u * sin[:, None] * way
        return y

    res, weights = [], []
    for x, w, dy in ((s["q"], s["wq"], s.get("dq")), (s["k"], s["wk"], s.get("dk"))):
        x, w = x.double(), w.double()
        norm = torch.sqrt((x ** 2).sum(-1, keepdim=True) / dim + EPS)
        if dy is None:
            res.append(rotated(x / norm * w, 1.0))
            continue
        z = rotated(dy.double(), -1.0)
        weights.append((z * x / norm).sum((0, 1)))
        z = z * w
        res.append(z / norm - x * (z * x).sum(-1, keepdim=True) / (dim * norm ** 3))
    return (*res, *weights)
