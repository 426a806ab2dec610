"""Operators of an attention block: head norms with the position rotation, and
causal attention over packed sequences, each with its gradient.

Thin wrappers over the calls of ``include/sync.h``: they check what a tensor
has that a pointer does not (device, type, shape), allocate outputs and pass
strides on.  Tensors are ``[rows, heads, dim]`` with the last dimension
contiguous; outputs are new contiguous tensors unless given.  Calls run on
the current stream, or on ``stream``; outputs that a call allocates belong to
the stream it runs on.
"""
from __future__ import annotations

import ctypes

import numpy as np

import paper_2608_13757_gb300 as _sg

BF16, FP16, FP32 = range(3)
_CODES = {}


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("row_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class NormRope(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("dim", ctypes.c_int32), ("rotated", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("eps", ctypes.c_float), ("q", Rows), ("k", Rows), ("q_weight", ctypes.c_void_p),
                ("k_weight", ctypes.c_void_p), ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p),
                ("n_positions", ctypes.c_int64), ("positions", ctypes.c_void_p)]


class AttnDesc(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("q_len", ctypes.POINTER(ctypes.c_int32)),
                ("k_len", ctypes.POINTER(ctypes.c_int32)), ("q_start", ctypes.POINTER(ctypes.c_int64)),
                ("k_start", ctypes.POINTER(ctypes.c_int64)), ("heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("train", ctypes.c_int32)]


class AttnSizes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("q_rows", "k_rows", "n_queries", "n_keys", "pairs", "device_bytes")] + [
        ("n_items", ctypes.c_int32), ("n_splits", ctypes.c_int32)]


def declare(lib: ctypes.CDLL):
    """Argument types of the library's calls that this module makes."""
    vp, P = ctypes.c_void_p, ctypes.POINTER
    rows = P(Rows)
    lib.sync_qk_norm_rope.argtypes = [P(NormRope), rows, rows, vp]
    lib.sync_qk_norm_rope_workspace.argtypes = [P(NormRope), P(ctypes.c_int64)]
    lib.sync_qk_norm_rope_backward.argtypes = [P(NormRope), rows, rows, rows, rows, vp, vp, vp, ctypes.c_int64, vp]
    lib.sync_attn_plan.argtypes = [P(AttnDesc), ctypes.c_int, P(vp)]
    lib.sync_attn_query.argtypes = [vp, P(AttnSizes)]
    lib.sync_attn_forward.argtypes = [vp, rows, rows, rows, ctypes.c_float, rows, vp, vp]
    lib.sync_attn_backward.argtypes = [vp, rows, rows, rows, rows, vp, rows, ctypes.c_float, rows, rows, rows, vp]
    lib.sync_attn_free.argtypes = [vp]
    lib.sync_attn_free.restype = None


def _code(dtype) -> int:
    if not _CODES:
        import torch
        _CODES.update({torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32})
    if dtype not in _CODES:
        raise _sg.SyncError(_sg.ERR_ARG, f"dtype must be bfloat16, float16 or float32, not {dtype}")
    return _CODES[dtype]


def _need(ok, what):
    if not ok:
        raise _sg.SyncError(_sg.ERR_ARG, what)


class _On:
    """The device of a call made current and its stream, for allocations too."""

    def __init__(self, device, stream):
        import torch
        self.device = torch.cuda.device(device)
        if stream is not None and not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(stream), device=device)
        self.given = stream
        self.scope = torch.cuda.stream(stream) if stream is not None else None

    def __enter__(self):
        import torch
        self.device.__enter__()
        if self.scope is not None:
            self.scope.__enter__()
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)

    def __exit__(self, *a):
        if self.scope is not None:
            self.scope.__exit__(*a)
        self.device.__exit__(*a)


def _rows(t, name, like=None, heads=None, dim=None) -> Rows:
    """A [rows, heads, dim] tensor's description; `like`: a tensor whose device
    and type it must have."""
    _need(t.dim() == 3, f"{name} must be [rows, heads, dim]")
    n, h, d = t.shape
    _need(t.is_cuda and (like is None or t.device == like.device), f"{name} must be on the call's GPU")
    _need(like is None or t.dtype == like.dtype, f"{name} must have the type of q")
    _need(heads is None or h == heads, f"{name} must have {heads} heads")
    _need(dim is None or d == dim, f"{name} must have heads of {dim} entries")
    rs, hs, ds = t.stride()
    _need(ds == 1 or d == 1 or n == 0, f"{name}: the entries of a head must be contiguous")
    # the stride of a dimension of size 1 is never used: pass a plain one
    if h == 1:
        hs = d
    if n <= 1:
        rs = h * d
    return Rows(t.data_ptr(), n, rs, hs)


def _vector(t, name, like, n, dtype):
    if t is None:
        return None
    _need(t.device == like.device and t.dtype == dtype, f"{name} must be {dtype} on the call's GPU")
    _need(t.numel() == n and t.is_contiguous(), f"{name} must be contiguous with {n} entries")
    return t.data_ptr()


def _norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved):
    import torch
    _need(q.dim() == 3 and k.dim() == 3, "q and k must be [rows, heads, dim]")
    n, heads, dim = q.shape
    p = NormRope()
    p.dtype, p.heads, p.kv_heads, p.dim = _code(q.dtype), heads, k.shape[1], dim
    p.q, p.k = _rows(q, "q"), _rows(k, "k", q, None, dim)
    p.eps, p.interleaved = eps, int(interleaved)
    p.q_weight = _vector(q_weight, "q_weight", q, dim, q.dtype)
    p.k_weight = _vector(k_weight, "k_weight", q, dim, q.dtype)
    _need(cos.dim() == 2 and cos.shape == sin.shape, "cos and sin must be [positions, rotated / 2]")
    p.rotated, p.n_positions = 2 * cos.shape[1], cos.shape[0]
    p.cos = _vector(cos, "cos", q, cos.numel(), torch.float32)
    p.sin = _vector(sin, "sin", q, sin.numel(), torch.float32)
    p.positions = _vector(positions, "positions", q, n, torch.int32)
    return p


def sync_qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions=None, eps: float = 1e-6,
                      interleaved: bool = False, out=None, stream=None):
    """Root-mean-square norm of every head of q and k, times its weights (or
    None), with the first 2 * cos.shape[1] entries of each head rotated by the
    angles of the token's position (int32; None: its row).  A position outside
    the table gives NaN.  Returns the pair of outputs; out=(q, k) works in place."""
    import torch
    p = _norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
    with _On(q.device, stream) as st:
        if out is None:
            out = (torch.empty(q.shape, dtype=q.dtype, device=q.device),
                   torch.empty(k.shape, dtype=q.dtype, device=q.device))
        _sg._check(_sg.lib().sync_qk_norm_rope(
            ctypes.byref(p), ctypes.byref(_rows(out[0], "out[0]", q, p.heads, p.dim)),
            ctypes.byref(_rows(out[1], "out[1]", q, p.kv_heads, p.dim)), st))
    return out


def sync_qk_norm_rope_backward(q, k, dq_out, dk_out, q_weight, k_weight, cos, sin, positions=None, eps: float = 1e-6,
                               interleaved: bool = False, out=None, stream=None):
    """(dq, dk, dq_weight, dk_weight) of sync_qk_norm_rope from its inputs and
    its outputs' gradients; a weight that is None has None.  out=(dq, dk) may
    be the outputs' gradients themselves."""
    import torch
    p = _norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
    with _On(q.device, stream) as st:
        if out is None:
            out = (torch.empty(q.shape, dtype=q.dtype, device=q.device),
                   torch.empty(k.shape, dtype=q.dtype, device=q.device))
        dw = [torch.empty(p.dim, dtype=q.dtype, device=q.device) if w is not None else None for w in (q_weight, k_weight)]
        need = ctypes.c_int64()
        _sg._check(_sg.lib().sync_qk_norm_rope_workspace(ctypes.byref(p), ctypes.byref(need)))
        work = torch.empty(need.value, dtype=torch.uint8, device=q.device)
        _sg._check(_sg.lib().sync_qk_norm_rope_backward(
            ctypes.byref(p), ctypes.byref(_rows(dq_out, "dq_out", q, p.heads, p.dim)),
            ctypes.byref(_rows(dk_out, "dk_out", q, p.kv_heads, p.dim)),
            ctypes.byref(_rows(out[0], "out[0]", q, p.heads, p.dim)),
            ctypes.byref(_rows(out[1], "out[1]", q, p.kv_heads, p.dim)),
            _sg._ptr(dw[0]), _sg._ptr(dw[1]), _sg._ptr(work), need.value, st))
    return out[0], out[1], dw[0], dw[1]


class AttnPlan:
    """The work of a packed batch on one GPU (owns device memory; freed on
    close / GC).  Calls on one plan must not overlap on the GPU."""

    def __init__(self, handle, device, heads, kv_heads, head_dim, dtype):
        self._h = handle
        self.device, self.heads, self.kv_heads, self.head_dim, self.dtype = device, heads, kv_heads, head_dim, dtype
        self.sizes = AttnSizes()
        _sg._check(_sg.lib().sync_attn_query(handle, ctypes.byref(self.sizes)))

    @property
    def handle(self):
        if not self._h:
            raise ValueError("plan already freed")
        return self._h

    def close(self):
        if self._h:
            _sg.lib().sync_attn_free(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def sync_attn_plan(q_lens, k_lens, heads: int, kv_heads: int, head_dim: int, dtype, q_starts=None, k_starts=None,
                   train: bool = False, device=None) -> AttnPlan:
    """Plan of a packed batch: sequence i has q_lens[i] queries, the last of the
    k_lens[i] tokens whose keys it attends to, causally.  Starts are rows of the
    query and key tensors (None: packed without gaps)."""
    import torch
    device = torch.cuda.current_device() if device is None else torch.device("cuda", device).index \
        if isinstance(device, int) else torch.device(device).index
    arrays = []
    for v, kind, name in ((q_lens, np.int32, "q_lens"), (k_lens, np.int32, "k_lens"), (q_starts, np.int64, "q_starts"),
                          (k_starts, np.int64, "k_starts")):
        if v is None:
            arrays.append(None)
            continue
        w = np.asarray(v, dtype=np.int64)
        _need(w.ndim == 1 and len(w) == len(q_lens), f"{name} must have one entry per sequence")
        _need(kind is np.int64 or w.size == 0 or (w.min() >= -1 << 31 and w.max() < 1 << 31), f"{name} must fit 32 bits")
        arrays.append(np.ascontiguousarray(w, dtype=kind))
    d = AttnDesc()
    d.n_seqs, d.heads, d.kv_heads, d.head_dim = len(q_lens), heads, kv_heads, head_dim
    d.dtype, d.train = _code(dtype), int(train)
    for (field, kind), a in zip((("q_len", ctypes.c_int32), ("k_len", ctypes.c_int32), ("q_start", ctypes.c_int64),
                                 ("k_start", ctypes.c_int64)), arrays):
        if a is not None:
            setattr(d, field, a.ctypes.data_as(ctypes.POINTER(kind)))
    h = ctypes.c_void_p()
    _sg._check(_sg.lib().sync_attn_plan(ctypes.byref(d), int(device), ctypes.byref(h)))
    return AttnPlan(h, torch.device("cuda", device), heads, kv_heads, head_dim, dtype)


def _attn_rows(plan, tensors):
    got = []
    for t, name, heads in tensors:
        _need(t.device == plan.device and t.dtype == plan.dtype, f"{name} must be {plan.dtype} on {plan.device}")
        got.append(_rows(t, name, None, heads, plan.head_dim))
    return [ctypes.byref(r) for r in got]


def _new(like_rows, heads, plan, covered):
    """An output: rows that no sequence has are zero."""
    import torch
    make = torch.empty if covered == like_rows else torch.zeros
    return make((like_rows, heads, plan.head_dim), dtype=plan.dtype, device=plan.device)


def sync_attn_forward(plan: AttnPlan, q, k, v, scale: float | None = None, out=None, lse=False, stream=None):
    """Causal attention of a planned batch.  With lse=True (or a float32 tensor
    [heads, rows of q] to write) returns (o, lse), as the gradient needs."""
    import torch
    scale = plan.head_dim ** -0.5 if scale is None else float(scale)
    with _On(plan.device, stream) as st:
        if out is None:
            out = _new(q.shape[0], plan.heads, plan, plan.sizes.n_queries)
        if lse is True:
            lse = torch.full((plan.heads, q.shape[0]), -float("inf"), dtype=torch.float32, device=plan.device) \
                if plan.sizes.n_queries != q.shape[0] else \
                torch.empty((plan.heads, q.shape[0]), dtype=torch.float32, device=plan.device)
        elif lse is False:
            lse = None
        if lse is not None:
            _vector(lse, "lse", q, plan.heads * q.shape[0], torch.float32)
        a = _attn_rows(plan, ((q, "q", plan.heads), (k, "k", plan.kv_heads), (v, "v", plan.kv_heads),
                              (out, "out", plan.heads)))
        _need(out.shape[0] == q.shape[0], "out must have the rows of q")
        _sg._check(_sg.lib().sync_attn_forward(plan.handle, a[0], a[1], a[2], scale, a[3], _sg._ptr(lse), st))
    return out if lse is None else (out, lse)


def sync_attn_backward(plan: AttnPlan, q, k, v, o, lse, do, scale: float | None = None, out=None, stream=None):
    """(dq, dk, dv) of sync_attn_forward, for a plan made with train=True."""
    import torch
    scale = plan.head_dim ** -0.5 if scale is None else float(scale)
    with _On(plan.device, stream) as st:
        _vector(lse, "lse", q, plan.heads * q.shape[0], torch.float32)
        if out is None:
            out = (_new(q.shape[0], plan.heads, plan, plan.sizes.n_queries),
                   _new(k.shape[0], plan.kv_heads, plan, plan.sizes.n_keys),
                   _new(k.shape[0], plan.kv_heads, plan, plan.sizes.n_keys))
        a = _attn_rows(plan, ((q, "q", plan.heads), (k, "k", plan.kv_heads), (v, "v", plan.kv_heads),
                              (o, "o", plan.heads), (do, "do", plan.heads), (out[0], "dq", plan.heads),
                              (out[1], "dk", plan.kv_heads), (out[2], "dv", plan.kv_heads)))
        _sg._check(_sg.lib().sync_attn_backward(plan.handle, a[0], a[1], a[2], a[3], _sg._ptr(lse), a[4], scale, a[5],
                                                a[6], a[7], st))
    return tuple(out)
