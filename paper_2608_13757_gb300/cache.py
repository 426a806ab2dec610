"""Rotation by positions with several axes, and a paged cache of keys and values
in 16 or 4 bits with the attention that reads it: an attention block's work
while it answers, token by token.

Thin wrappers over the calls of ``include/sync.h``, in the manner of
``attention``: tensors are ``[rows, heads, dim]``, calls run on the current
stream or on ``stream``, nothing is recorded for autograd.  The lengths, row
starts and page tables of a step are int32 tensors on the GPU that the kernels
read: no call waits for the device, and a captured call follows what they hold
when it is replayed.
"""
from __future__ import annotations

import ctypes

import paper_2608_13757_gb300 as _sg
from .attention import _On, Rows, _code, _current_stream, _need, _not_recorded, _rows, _vector


SHORT = 128      # tokens of max_pages pages up to which attention takes no workspace


class Rotation(ctypes.Structure):
    _fields_ = [("rotated", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("n_axes", ctypes.c_int32),
                ("pair_axis", ctypes.c_char_p), ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p),
                ("n_positions", ctypes.c_int64), ("positions", ctypes.c_void_p), ("position_stride", ctypes.c_int64)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("dim", ctypes.c_int32), ("q", Rows), ("k", Rows), ("turn", Rotation)]


class CacheDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "bits", "kv_heads", "head_dim", "page", "n_pages")] + [
        (n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")]


class CacheSeqs(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("page_table", ctypes.c_void_p),
                ("table_stride", ctypes.c_int64), ("lens", ctypes.c_void_p), ("row_starts", ctypes.c_void_p)]


def declare(lib: ctypes.CDLL):
    """Argument types of the library's calls that this module makes."""
    vp, P, i32 = ctypes.c_void_p, ctypes.POINTER, ctypes.c_int32
    rows, cache, seqs = P(Rows), P(CacheDesc), P(CacheSeqs)
    lib.sync_rope.argtypes = lib.sync_rope_backward.argtypes = [P(RopeDesc), rows, rows, vp]
    lib.sync_cache_append.argtypes = [cache, seqs, rows, rows, i32, rows, rows, P(Rotation), i32, vp]
    lib.sync_cache_read.argtypes = [cache, seqs, rows, rows, i32, vp]
    lib.sync_cache_attn_workspace.argtypes = [cache, i32, i32, P(ctypes.c_int64)]
    lib.sync_cache_attn.argtypes = [cache, seqs, i32, rows, ctypes.c_float, i32, rows, vp, i32, vp, ctypes.c_int64, vp]


def _current_device() -> int:
    """torch.cuda.current_device() where a GPU is in use already."""
    import torch
    return torch._C._cuda_getDevice()


def _rotation(cos, sin, positions, axes, interleaved, n, device) -> Rotation:
    """The description of a rotation of n rows."""
    import torch
    shape = cos.shape
    if len(shape) != 2 or shape != sin.shape:
        _need(False, "cos and sin must be [positions, rotated / 2]")
    n_pos, half = shape
    n_axes, at, stride = 1, None, n
    if positions is not None:
        if positions.dtype is not torch.int32 or positions.get_device() != device:
            _need(False, f"positions must be int32 on GPU {device}")
        if positions.dim() == 2:
            n_axes, stride = positions.shape[0], positions.stride(0)
        rows = positions.shape[-1] if positions.dim() in (1, 2) else -1
        if rows != n or n > 1 and positions.stride(-1) != 1:
            _need(False, "positions must be [rows] or [axes, rows], the rows contiguous")
        at = positions.data_ptr()
    if axes is not None:
        _need(len(axes) == half, "axes must name an axis for every pair")
        try:
            axes = bytes(axes if isinstance(axes, (bytes, list, tuple)) else list(axes))
        except (TypeError, ValueError):
            _need(False, "axes must be whole numbers from 0 on")
    else:
        _need(n_axes == 1, "positions of several axes need axes")
    return Rotation(2 * half, bool(interleaved), n_axes, axes, _vector(cos, "cos", device, n_pos * half, torch.float32),
                    _vector(sin, "sin", device, n_pos * half, torch.float32), n_pos, at, stride)


def _rope(name, f, q, k, cos, sin, positions, axes, interleaved, out, stream):
    import torch
    if stream is not None:
        with _On(q.device, stream):
            return _rope(name, f, q, k, cos, sin, positions, axes, interleaved, out, None)
    _need(q.dim() == 3 and k.dim() == 3, "q and k must be [rows, heads, dim]")
    _need(q.is_cuda, "q must be on a GPU")
    device, dtype = q.get_device(), q.dtype
    if _current_device() != device:
        with torch.cuda.device(device):
            return _rope(name, f, q, k, cos, sin, positions, axes, interleaved, out, None)
    n, heads, dim = q.shape
    kv = k.shape[1]
    p = RopeDesc(_code(dtype), heads, kv, dim, _rows(q, "q", dtype, device, heads, dim),
                 _rows(k, "k", dtype, device, kv, dim), _rotation(cos, sin, positions, axes, interleaved, n, device))
    if out is None:
        where = q.device
        out = torch.empty((n, heads, dim), dtype=dtype, device=where), torch.empty((k.shape[0], kv, dim), dtype=dtype, device=where)
    _sg._check(f(p, _rows(out[0], "out[0]", dtype, device, heads, dim), _rows(out[1], "out[1]", dtype, device, kv, dim),
                 _current_stream(device)))
    return tuple(out)


def sync_rope(q, k, cos, sin, positions=None, axes=None, interleaved: bool = False, out=None, stream=None):
    """Rotation of every head of q and k: the pairs (j, j + half), or (2j, 2j + 1)
    when interleaved, of the first 2 * half entries by the angles of the tables cos
    and sin (float32 [positions, half]).  positions: int32 [rows] (None: the row), or
    [axes, rows] with axes[j] naming the axis that turns pair j, as for a video's
    tokens in time, height and width.  A position outside the table gives NaN.
    Returns the pair of outputs; out=(q, k) works in place."""
    if q.requires_grad or k.requires_grad:
        _not_recorded("sync_rope")
    return _rope("sync_rope", _sg.lib().sync_rope, q, k, cos, sin, positions, axes, interleaved, out, stream)


def sync_rope_backward(dq_out, dk_out, cos, sin, positions=None, axes=None, interleaved: bool = False, out=None,
                       stream=None):
    """(dq, dk) of sync_rope from its outputs' gradients: the rotation back.
    out may be the outputs' gradients themselves."""
    return _rope("sync_rope_backward", _sg.lib().sync_rope_backward, dq_out, dk_out, cos, sin, positions, axes,
                 interleaved, out, stream)


class KVCache:
    """Pages of keys and values on one GPU: k and v, with bits=4 their k_scale and
    v_scale too (the layout is sync_cache's in include/sync.h).  What pages hold
    before they are written is undefined, and never read."""

    def __init__(self, n_pages, page, kv_heads, head_dim, dtype, bits, device):
        import torch
        self.n_pages, self.page, self.kv_heads, self.head_dim = n_pages, page, kv_heads, head_dim
        self.dtype, self.bits, self.device, self.index = dtype, bits, device, device.index
        shape = (n_pages, kv_heads, page)
        self.k_scale = self.v_scale = None
        if bits == 16:
            self.k, self.v = (torch.empty(shape + (head_dim,), dtype=dtype, device=device) for _ in range(2))
        else:
            self.k, self.v = (torch.empty(shape + (head_dim // 2,), dtype=torch.uint8, device=device) for _ in range(2))
            self.k_scale, self.v_scale = (torch.empty(shape + (head_dim // 32,), dtype=torch.float16, device=device) for _ in range(2))
        self.desc = CacheDesc(_code(dtype), bits, kv_heads, head_dim, page, n_pages, self.k.data_ptr(), self.v.data_ptr(),
                              _sg._ptr(self.k_scale), _sg._ptr(self.v_scale))
        self._work = {}                # workspace bytes of (heads, max_new)

    def workspace(self, heads: int, max_new: int) -> int:
        """Bytes of workspace of an attention call."""
        n = self._work.get((heads, max_new))
        if n is None:
            need = ctypes.c_int64()
            _sg._check(_sg.lib().sync_cache_attn_workspace(self.desc, heads, max_new, need))
            n = self._work[heads, max_new] = need.value
        return n


def sync_kv_cache(n_pages: int, page: int, kv_heads: int, head_dim: int, dtype, bits: int = 16, device=None) -> KVCache:
    """A cache of n_pages pages of `page` tokens (a power of two from 16 on) for
    one layer, its keys and values held in dtype (bits=16) or in 4 bits with a
    float16 scale for every 32 entries (head_dim a multiple of 32 then)."""
    import torch
    where = torch.device("cuda" if device is None else device if not isinstance(device, int) else f"cuda:{device}")
    _need(where.type == "cuda", f"device must be a GPU, not {where}")
    _need(all(isinstance(x, int) for x in (n_pages, page, kv_heads, head_dim, bits)), "sizes must be whole numbers")
    need = ctypes.c_int64()
    _sg._check(_sg.lib().sync_cache_attn_workspace(CacheDesc(_code(dtype), bits, kv_heads, head_dim, page, n_pages),
                                                   kv_heads, 1, need))
    if where.index is None:
        where = torch.device("cuda", torch.cuda.current_device())
    return KVCache(n_pages, page, kv_heads, head_dim, dtype, bits, where)


def _seqs(page_table, lens, row_starts, device) -> CacheSeqs:
    import torch
    i32 = torch.int32
    n = lens.shape[0] if lens.dim() == 1 else -1
    if page_table.dim() != 2 or page_table.shape[0] != n or page_table.dtype is not i32 or page_table.get_device() != device:
        _need(n >= 0, "lens must be [sequences]")
        _need(False, f"page_table must be int32 [sequences, pages] on GPU {device}")
    width = page_table.shape[1]
    if width > 1 and n and page_table.stride(1) != 1:
        _need(False, "the pages of a sequence must be contiguous in page_table")
    return CacheSeqs(n, width, page_table.data_ptr(), page_table.stride(0), _vector(lens, "lens", device, n, i32),
                     _vector(row_starts, "row_starts", device, n + 1, i32))


def sync_cache_append(cache: KVCache, k, v, page_table, lens, row_starts=None, q=None, cos=None, sin=None,
                      positions=None, axes=None, interleaved: bool = False, out=None, stream=None):
    """Writes a step's new keys, turned, and values to the cache, and returns the
    step's queries q, turned (None without q; out=q works in place).

    page_table: int32 [sequences, pages], the pages of every sequence in order;
    lens: int32 [sequences], their tokens with the new ones; row_starts: int32
    [sequences + 1], the first row of each in k, v and q, rows before the first and
    past the last being padding (None: one row each).  cos, sin, positions, axes and interleaved are
    sync_rope's, positions None meaning a token's place in its sequence; without
    cos and sin nothing is turned."""
    import torch
    if stream is not None:
        with _On(cache.device, stream):
            return sync_cache_append(cache, k, v, page_table, lens, row_starts, q, cos, sin, positions, axes, interleaved, out)
    device, dtype, kv, dim = cache.index, cache.dtype, cache.kv_heads, cache.head_dim
    if _current_device() != device:
        with torch.cuda.device(device):
            return sync_cache_append(cache, k, v, page_table, lens, row_starts, q, cos, sin, positions, axes, interleaved, out)
    a, b = _rows(k, "k", dtype, device, kv, dim), _rows(v, "v", dtype, device, kv, dim)
    if k.requires_grad or v.requires_grad or q is not None and q.requires_grad:
        _not_recorded("sync_cache_append", backward=False)
    _need((cos is None) == (sin is None), "cos and sin must both be given or both be None")
    turn = None if cos is None else _rotation(cos, sin, positions, axes, interleaved, a.rows, device)
    heads, given, to, fill = 0, None, None, False
    if q is not None:
        heads = q.shape[1] if q.dim() == 3 else 0
        given = _rows(q, "q", dtype, device, heads, dim)
        if out is None:
            out, fill = torch.empty((a.rows, heads, dim), dtype=dtype, device=cache.device), True
        to = _rows(out, "out", dtype, device, heads, dim)
    _sg._check(_sg.lib().sync_cache_append(cache.desc, _seqs(page_table, lens, row_starts, device), a, b, heads, given, to,
                                           turn, fill, _current_stream(device)))
    return out if q is not None else None


def sync_cache_read(cache: KVCache, page_table, lens, row_starts, rows: int | None = None, out=None, stream=None):
    """(k, v): the cached tokens of every sequence as packed rows [rows, kv_heads,
    head_dim] of the cache's dtype, sequence s in rows row_starts[s] ..
    row_starts[s + 1] - 1, as sync_attn_forward takes them for the next piece of a
    prompt.  out=(k, v): tensors to write instead of new ones of `rows` rows."""
    import torch
    if stream is not None:
        with _On(cache.device, stream):
            return sync_cache_read(cache, page_table, lens, row_starts, rows, out)
    device, dtype, kv, dim = cache.index, cache.dtype, cache.kv_heads, cache.head_dim
    if _current_device() != device:
        with torch.cuda.device(device):
            return sync_cache_read(cache, page_table, lens, row_starts, rows, out)
    _need(row_starts is not None, "row_starts must be given")
    fill = out is None
    if fill:
        _need(isinstance(rows, int) and rows >= 0, "rows must be a whole number from 0 on, or out given")
        out = tuple(torch.empty((rows, kv, dim), dtype=dtype, device=cache.device) for _ in range(2))
    _sg._check(_sg.lib().sync_cache_read(cache.desc, _seqs(page_table, lens, row_starts, device),
                                         _rows(out[0], "out[0]", dtype, device, kv, dim),
                                         _rows(out[1], "out[1]", dtype, device, kv, dim), fill, _current_stream(device)))
    return tuple(out)


def sync_cache_attn(cache: KVCache, q, page_table, lens, row_starts=None, max_new: int = 1, scale: float | None = None,
                    out=None, lse=False, stream=None):
    """Attention of a step's rows over the cache, after sync_cache_append (whose
    page_table, lens and row_starts it takes): row i of the n rows of a sequence
    sees its tokens 0 .. lens - n + i.  max_new: the most rows that a sequence has,
    for the choice of the tile.  With lse=True (or a float32 tensor [heads, rows] to
    write) returns (o, lse)."""
    import torch
    if stream is not None:
        with _On(cache.device, stream):
            return sync_cache_attn(cache, q, page_table, lens, row_starts, max_new, scale, out, lse)
    device, dtype, dim = cache.index, cache.dtype, cache.head_dim
    if _current_device() != device:
        with torch.cuda.device(device):
            return sync_cache_attn(cache, q, page_table, lens, row_starts, max_new, scale, out, lse)
    heads = q.shape[1] if q.dim() == 3 else 0
    a = _rows(q, "q", dtype, device, heads, dim)
    if q.requires_grad:
        _not_recorded("sync_cache_attn", backward=False)
    n = a.rows
    fill = out is None
    if fill:
        out = torch.empty((n, heads, dim), dtype=dtype, device=cache.device)
    if lse is True:
        lse = torch.empty((heads, n), dtype=torch.float32, device=cache.device)
        if not fill and row_starts is not None:
            lse.fill_(-float("inf"))
    at = None if lse is False or lse is None else _vector(lse, "lse", device, heads * n, torch.float32)
    work, size = None, 0
    if page_table.shape[-1] * cache.page > SHORT:
        size = cache.workspace(heads, max_new)
        work = torch.empty(size, dtype=torch.uint8, device=cache.device)
    _sg._check(_sg.lib().sync_cache_attn(cache.desc, _seqs(page_table, lens, row_starts, device), heads, a,
                                         dim ** -0.5 if scale is None else scale, max_new,
                                         _rows(out, "out", dtype, device, heads, dim), at, fill,
                                         None if work is None else work.data_ptr(), size, _current_stream(device)))
    return out if at is None and not isinstance(lse, torch.Tensor) else (out, lse)
