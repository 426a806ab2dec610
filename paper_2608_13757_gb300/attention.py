"""Operators of an attention block: head norms with the position rotation, and
causal attention over packed sequences, each with its gradient.

Thin wrappers over the calls of ``include/sync.h``: they check what a tensor
has that a pointer does not (device, type, shape), allocate outputs and pass
strides on.  Tensors are ``[rows, heads, dim]`` with the last dimension
contiguous; outputs are new contiguous tensors unless given.  Calls run on
the current stream, or on ``stream``; outputs that a call allocates belong to
the stream it runs on.  Inputs that belong to another one are the caller's to
order and to keep until the call is done (``Tensor.record_stream``).

Nothing is recorded for autograd: outputs carry no gradient, and the gradients
are calls of their own.  A forward call warns of inputs that require one while
gradients are recorded.
"""
from __future__ import annotations

import ctypes
import warnings

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
    lib.sync_attn_status.argtypes = [vp]
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


def _not_recorded(name):
    """Says that a call drops the gradient that an input of it requires."""
    import torch
    if torch.is_grad_enabled():
        warnings.warn(f"{name} records nothing for autograd: its outputs carry no gradient to the inputs that require one "
                      f"(use {name.replace('_forward', '')}_backward, and torch.no_grad() around this call)", stacklevel=3)


def _current_stream(device: int) -> int:
    """The current stream's handle, without the object around it (a microsecond)."""
    import torch
    return torch._C._cuda_getCurrentRawStream(device)


class _On:
    """The stream of a call that names one, current for allocations too.  (A
    call that names none takes the current stream of its device directly.)"""

    def __init__(self, device, stream):
        import torch
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(stream), device=device)
        self.stream, self.scope = stream, torch.cuda.stream(stream)

    def __enter__(self):
        self.scope.__enter__()
        return self.stream.cuda_stream

    def __exit__(self, *a):
        self.scope.__exit__(*a)


def _rows(t, name, dtype, device, heads, dim) -> Rows:
    """A [rows, heads, dim] tensor's description, checked against the call's."""
    shape = t.shape
    if len(shape) != 3 or t.dtype is not dtype or t.get_device() != device:
        _need(len(shape) == 3, f"{name} must be [rows, heads, dim]")
        _need(False, f"{name} must be {dtype} on GPU {device}")
    n, h, d = shape
    rs, hs, ds = t.stride()
    if h != heads or d != dim or ds != 1:
        _need(h == heads and d == dim, f"{name} must have {heads} heads of {dim} entries")
        _need(n == 0, f"{name}: the entries of a head must be contiguous")
    # the stride of a dimension of size 1 is never used: pass a plain one
    return Rows(t.data_ptr(), n, rs if n > 1 else h * d, hs if h > 1 else d)


def _vector(t, name, device, n, dtype):
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != device or t.numel() != n or not t.is_contiguous():
        _need(False, f"{name} must be contiguous {dtype} with {n} entries on GPU {device}")
    return t.data_ptr()


def _norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved):
    import torch
    if q.dim() != 3 or k.dim() != 3 or cos.dim() != 2 or cos.shape != sin.shape or not q.is_cuda:
        _need(q.dim() == 3 and k.dim() == 3, "q and k must be [rows, heads, dim]")
        _need(q.is_cuda, "q must be on a GPU")
        _need(False, "cos and sin must be [positions, rotated / 2]")
    n, heads, dim = q.shape
    dtype, device, kv_heads, (n_pos, half) = q.dtype, q.get_device(), k.shape[1], cos.shape
    return NormRope(_code(dtype), heads, kv_heads, dim, 2 * half, bool(interleaved), eps,
                    _rows(q, "q", dtype, device, heads, dim), _rows(k, "k", dtype, device, kv_heads, dim),
                    _vector(q_weight, "q_weight", device, dim, dtype), _vector(k_weight, "k_weight", device, dim, dtype),
                    _vector(cos, "cos", device, n_pos * half, torch.float32),
                    _vector(sin, "sin", device, n_pos * half, torch.float32), n_pos,
                    _vector(positions, "positions", device, n, torch.int32))


def sync_qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions=None, eps: float = 1e-6,
                      interleaved: bool = False, out=None, stream=None):
    """Root-mean-square norm of every head of q and k, times its weights (or
    None), with the first 2 * cos.shape[1] entries of each head rotated by the
    angles of the token's position (int32; None: its row).  A position outside
    the table gives NaN; where nothing is rotated (tables of width 0, of any
    length) positions are not looked at.  Returns the pair of outputs; out=(q, k) works in place."""
    import torch
    if stream is not None:
        with _On(q.device, stream):
            return sync_qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, out)
    p = _norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
    device, dtype = q.get_device(), q.dtype
    if torch.cuda.current_device() != device:
        with torch.cuda.device(device):
            return sync_qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, out)
    if q.requires_grad or k.requires_grad or q_weight is not None and q_weight.requires_grad or \
            k_weight is not None and k_weight.requires_grad:
        _not_recorded("sync_qk_norm_rope")
    if out is None:
        where = q.device
        out = torch.empty(q.shape, dtype=dtype, device=where), torch.empty(k.shape, dtype=dtype, device=where)
    _sg._check(_sg.lib().sync_qk_norm_rope(p, _rows(out[0], "out[0]", dtype, device, p.heads, p.dim),
                                           _rows(out[1], "out[1]", dtype, device, p.kv_heads, p.dim),
                                           _current_stream(device)))
    return out


def sync_qk_norm_rope_backward(q, k, dq_out, dk_out, q_weight, k_weight, cos, sin, positions=None, eps: float = 1e-6,
                               interleaved: bool = False, out=None, stream=None):
    """(dq, dk, dq_weight, dk_weight) of sync_qk_norm_rope from its inputs and
    its outputs' gradients; a weight that is None has None.  out=(dq, dk) may
    be the outputs' gradients themselves."""
    import torch
    if stream is not None:
        with _On(q.device, stream):
            return sync_qk_norm_rope_backward(q, k, dq_out, dk_out, q_weight, k_weight, cos, sin, positions, eps,
                                              interleaved, out)
    p = _norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
    device, dtype = q.get_device(), q.dtype
    if torch.cuda.current_device() != device:
        with torch.cuda.device(device):
            return sync_qk_norm_rope_backward(q, k, dq_out, dk_out, q_weight, k_weight, cos, sin, positions, eps,
                                              interleaved, out)
    if out is None:
        where = q.device
        out = torch.empty(q.shape, dtype=dtype, device=where), torch.empty(k.shape, dtype=dtype, device=where)
    heads, kv, dim = p.heads, p.kv_heads, p.dim
    a = (_rows(dq_out, "dq_out", dtype, device, heads, dim), _rows(dk_out, "dk_out", dtype, device, kv, dim),
         _rows(out[0], "out[0]", dtype, device, heads, dim), _rows(out[1], "out[1]", dtype, device, kv, dim))
    dwq = torch.empty(dim, dtype=dtype, device=q.device) if q_weight is not None else None
    dwk = torch.empty(dim, dtype=dtype, device=q.device) if k_weight is not None else None
    need = ctypes.c_int64()
    _sg._check(_sg.lib().sync_qk_norm_rope_workspace(p, need))
    work = torch.empty(need.value, dtype=torch.uint8, device=q.device)
    _sg._check(_sg.lib().sync_qk_norm_rope_backward(p, *a, _sg._ptr(dwq), _sg._ptr(dwk), work.data_ptr(), need.value,
                                                    _current_stream(device)))
    return out[0], out[1], dwq, dwk


# Handles of plans that were dropped without close().  Freeing one waits for the
# device and would invalidate a capture, and a finaliser may run anywhere: it
# only leaves the handle here, for the next sync_attn_plan.
_dropped = []


class AttnPlan:
    """The work of a packed batch on one GPU.  Owns device memory, which close()
    frees, waiting for the device; that of a plan that is dropped instead is
    freed by the next sync_attn_plan.  Keep it as long as a graph that captured
    its calls.  Calls on one plan must not overlap on the GPU."""

    def __init__(self, handle, device, heads, kv_heads, head_dim, dtype):
        self._h = handle
        self.device, self.heads, self.kv_heads, self.head_dim, self.dtype = device, heads, kv_heads, head_dim, dtype
        self.index, self.sizes = device.index, AttnSizes()
        _sg._check(_sg.lib().sync_attn_query(handle, ctypes.byref(self.sizes)))
        self.n_queries, self.n_keys = self.sizes.n_queries, self.sizes.n_keys

    @property
    def handle(self):
        if not self._h:
            raise ValueError("plan already freed")
        return self._h

    def check(self):
        """Raises if a kernel of a call on this plan that is done on the GPU gave
        up waiting, so that its results are not valid.  (Synchronise first; the
        plan's later calls raise too.)"""
        _sg._check(_sg.lib().sync_attn_status(self.handle))

    def close(self):
        if self._h:
            _sg.lib().sync_attn_free(self._h)
            self._h = None

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h and _dropped is not None:      # (None while the interpreter ends)
            _dropped.append(h)


def sync_attn_plan(q_lens, k_lens, heads: int, kv_heads: int, head_dim: int, dtype, q_starts=None, k_starts=None,
                   train: bool = False, device=None) -> AttnPlan:
    """Plan of a packed batch: sequence i has q_lens[i] queries, the last of the
    k_lens[i] tokens whose keys it attends to, causally.  Starts are rows of the
    query and key tensors (None: packed without gaps)."""
    import torch
    index = device if device is None or isinstance(device, int) else torch.device(device)
    if isinstance(index, torch.device):
        _need(index.type == "cuda", f"device must be a GPU, not {index}")
        index = index.index
    if index is None:
        index = torch.cuda.current_device()
    arrays = []
    for v, kind, name in ((q_lens, np.int32, "q_lens"), (k_lens, np.int32, "k_lens"), (q_starts, np.int64, "q_starts"),
                          (k_starts, np.int64, "k_starts")):
        if v is None:
            arrays.append(None)
            continue
        given = np.asarray(v)
        if given.dtype.kind == "f":
            _need(bool(np.all(np.isfinite(given) & (given == np.floor(given)))), f"{name} must be whole numbers")
        w = given.astype(np.int64)
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
    try:
        while True:
            _sg.lib().sync_attn_free(_dropped.pop())
    except IndexError:                      # none left (another thread may have taken the last)
        pass
    h = ctypes.c_void_p()
    _sg._check(_sg.lib().sync_attn_plan(ctypes.byref(d), index, ctypes.byref(h)))
    return AttnPlan(h, torch.device("cuda", index), heads, kv_heads, head_dim, dtype)


def _new(rows, heads, plan, covered):
    """An output: rows that no sequence has are zero."""
    import torch
    make = torch.empty if covered == rows else torch.zeros
    return make((rows, heads, plan.head_dim), dtype=plan.dtype, device=plan.device)


def sync_attn_forward(plan: AttnPlan, q, k, v, scale: float | None = None, out=None, lse=False, stream=None):
    """Causal attention of a planned batch.  With lse=True (or a float32 tensor
    [heads, rows of q] to write) returns (o, lse), as the gradient needs."""
    import torch
    if stream is not None:
        with _On(plan.device, stream):
            return sync_attn_forward(plan, q, k, v, scale, out, lse)
    dtype, device, heads, kv, dim = plan.dtype, plan.index, plan.heads, plan.kv_heads, plan.head_dim
    a = (_rows(q, "q", dtype, device, heads, dim), _rows(k, "k", dtype, device, kv, dim),
         _rows(v, "v", dtype, device, kv, dim))
    if q.requires_grad or k.requires_grad or v.requires_grad:
        _not_recorded("sync_attn_forward")
    n = q.shape[0]
    if out is None:
        out = _new(n, heads, plan, plan.n_queries)
    o = _rows(out, "out", dtype, device, heads, dim)
    if o.rows != n:
        _need(False, "out must have the rows of q")
    if lse is True:
        lse = torch.empty((heads, n), dtype=torch.float32, device=plan.device)
        if plan.n_queries != n:
            lse.fill_(-float("inf"))
    at = None if lse is False or lse is None else _vector(lse, "lse", device, heads * n, torch.float32)
    _sg._check(_sg.lib().sync_attn_forward(plan.handle, *a, dim ** -0.5 if scale is None else scale, o, at,
                                           _current_stream(device)))
    return out if at is None and not isinstance(lse, torch.Tensor) else (out, lse)


def sync_attn_backward(plan: AttnPlan, q, k, v, o, lse, do, scale: float | None = None, out=None, stream=None):
    """(dq, dk, dv) of sync_attn_forward, for a plan made with train=True."""
    import torch
    if stream is not None:
        with _On(plan.device, stream):
            return sync_attn_backward(plan, q, k, v, o, lse, do, scale, out)
    dtype, device, heads, kv, dim = plan.dtype, plan.index, plan.heads, plan.kv_heads, plan.head_dim
    a = (_rows(q, "q", dtype, device, heads, dim), _rows(k, "k", dtype, device, kv, dim),
         _rows(v, "v", dtype, device, kv, dim), _rows(o, "o", dtype, device, heads, dim))
    g = _rows(do, "do", dtype, device, heads, dim)
    n, m = q.shape[0], k.shape[0]
    at = _vector(lse, "lse", device, heads * n, torch.float32)
    if out is None:
        out = (_new(n, heads, plan, plan.n_queries), _new(m, kv, plan, plan.n_keys),
               _new(m, kv, plan, plan.n_keys))
    d = (_rows(out[0], "dq", dtype, device, heads, dim), _rows(out[1], "dk", dtype, device, kv, dim),
         _rows(out[2], "dv", dtype, device, kv, dim))
    _sg._check(_sg.lib().sync_attn_backward(plan.handle, *a, at, g, dim ** -0.5 if scale is None else scale, *d,
                                            _current_stream(device)))
    return tuple(out)
