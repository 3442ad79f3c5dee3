"""A paged cache of keys and values, operations on its pages, and the attention of decoding requests over it.

:class:`Cache` holds the caller's tensors; the functions enqueue kernels on the current (or the given) stream and
return without waiting; a given stream is not ordered against the current one, and what a call reads there (lists and
new rows too) is kept by the caller until it has run.  The rules are those of ``bdlm_cache_*`` and ``bdlm_prefix_attn`` in
``include/bdlm_attn.h``.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import _dtype_code, _expect, _launch, _made, lib
from .packed import _int, _Rows, _rows, _workspace

__all__ = ["Cache", "cache_new", "cache_grow", "cache_write", "cache_fork", "cache_free", "cache_compact",
           "prefix_attn", "prefix_attn_workspace_bytes", "CACHE_OK", "CACHE_BAD_LIST", "CACHE_NO_PAGES"]

CACHE_OK, CACHE_BAD_LIST, CACHE_NO_PAGES = 0, 1, 2


class _Cache(ctypes.Structure):  # bdlm_cache
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "table", "lens", "refs", "status", "work")] + \
               [(n, ctypes.c_int64) for n in ("layers", "pages", "page_size", "seqs", "max_pages")] + \
               [(n, ctypes.c_int32) for n in ("kv_heads", "head_dim", "dtype", "reserved")]


def declare(L: ctypes.CDLL):
    vp, i64, i32, sz, cp = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t, ctypes.POINTER(_Cache)
    L.bdlm_cache_work_bytes.argtypes = [i64, i64]
    L.bdlm_cache_work_bytes.restype = sz
    L.bdlm_cache_grow.argtypes = [cp, i64, vp, vp, vp]
    L.bdlm_cache_fork.argtypes = [cp, i64, vp, vp, vp]
    L.bdlm_cache_free.argtypes = [cp, i64, vp, vp]
    L.bdlm_cache_compact.argtypes = [cp, vp]
    L.bdlm_cache_write.argtypes = [cp, i64, i64, vp, vp, vp, i64, _Rows, _Rows, vp]
    L.bdlm_prefix_attn_workspace_bytes.argtypes = [cp, i64, i64, i32, i64]
    L.bdlm_prefix_attn_workspace_bytes.restype = sz
    L.bdlm_prefix_attn.argtypes = [cp, i64, i64, vp, i64, i32, i64, i32, ctypes.c_float, vp, vp, vp, vp, sz, vp]
    for name in ("grow", "fork", "free", "compact", "write"):
        getattr(L, "bdlm_cache_" + name).restype = ctypes.c_int
    L.bdlm_prefix_attn.restype = ctypes.c_int


class Cache:
    """A paged cache over the caller's tensors (all on one GPU, contiguous):

    ``k``, ``v``  ``[layers][pages][page_size][kv_heads][head_dim]``, bf16 or fp32
    ``table``     ``[seqs][max_pages]`` int32: the pages of a sequence in order, -1 behind them
    ``lens``      ``[seqs]`` int32: tokens
    ``refs``      ``[pages]`` int32: tables that hold a page, 0 for free ones
    ``status``    ``[2]`` int32: ``CACHE_*`` of the last page operation, and the pages it lacked
    """

    def __init__(self, k, v, table, lens, refs, status):
        if not isinstance(k, torch.Tensor) or k.dim() != 5:
            raise ValueError("k must be a [layers][pages][page_size][kv_heads][head_dim] tensor")
        if not isinstance(table, torch.Tensor) or table.dim() != 2:
            raise ValueError("table must be a [seqs][max_pages] tensor")
        code = _dtype_code(k.dtype)
        layers, pages, page_size, kv_heads, head_dim = k.shape
        seqs, max_pages = table.shape
        _expect("k", k, k.dtype, k.shape)
        _expect("v", v, k.dtype, k.shape)
        _expect("table", table, torch.int32, table.shape)
        _expect("lens", lens, torch.int32, (seqs,))
        _expect("refs", refs, torch.int32, (pages,))
        _expect("status", status, torch.int32, (2,))
        for name, t in (("v", v), ("table", table), ("lens", lens), ("refs", refs), ("status", status)):
            if t.device != k.device:
                raise ValueError(f"{name} must be on {k.device}, got {t.device}")
        self.k, self.v, self.table, self.lens, self.refs, self.status = k, v, table, lens, refs, status
        self.layers, self.pages, self.page_size, self.kv_heads, self.head_dim = k.shape
        self.seqs, self.max_pages = seqs, max_pages
        self.dtype, self.device, self.gpu = k.dtype, k.device, k.get_device()
        nbytes = lib().bdlm_cache_work_bytes(pages, seqs)
        self._work = torch.empty(max(64, nbytes) // 4, dtype=torch.int32, device=k.device)
        self._record = _Cache(k.data_ptr(), v.data_ptr(), table.data_ptr(), lens.data_ptr(), refs.data_ptr(),
                              status.data_ptr(), self._work.data_ptr(), layers, pages, page_size, seqs, max_pages,
                              kv_heads, head_dim, code, 0)
        self._ref = ctypes.byref(self._record)
        self._tensors, self._streams = (k, v, table, lens, refs, status, self._work), set()

    def __repr__(self):
        return (f"Cache(layers={self.layers}, pages={self.pages} x {self.page_size}, seqs={self.seqs} x {self.max_pages} "
                f"pages, kv_heads={self.kv_heads}, head_dim={self.head_dim}, {self.dtype}, {self.device})")


def cache_new(layers: int, pages: int, page_size: int, kv_heads: int, head_dim: int, seqs: int, max_pages: int,
              dtype=torch.bfloat16, device="cuda") -> Cache:
    """An empty cache: every page free, every sequence without tokens."""
    shape = (layers, pages, page_size, kv_heads, head_dim)
    i32 = dict(dtype=torch.int32, device=device)
    return Cache(torch.zeros(shape, dtype=dtype, device=device), torch.zeros(shape, dtype=dtype, device=device),
                 torch.full((seqs, max_pages), -1, **i32), torch.zeros(seqs, **i32), torch.zeros(pages, **i32),
                 torch.zeros(2, **i32))


def _cache(c):
    if not isinstance(c, Cache):
        raise TypeError(f"cache must be a Cache, got {type(c).__name__}")
    return c


def _list(c, name, t, n=None):
    """An int32 list on the cache's device: its address."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor, got {type(t).__name__}")
    if t.dtype is not torch.int32:
        raise TypeError(f"{name} must be torch.int32, got {t.dtype}")
    shape = t.shape
    if len(shape) != 1 or (n is not None and shape[0] != n):
        raise ValueError(f"{name} must have shape ({'n' if n is None else n},), got {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.get_device() != c.gpu:
        raise ValueError(f"{name} must be on {c.device}, got {t.device}")
    return t.data_ptr()


def cache_grow(cache: Cache, seqs, counts, stream=None):
    """Room for ``counts[i]`` more tokens of sequence ``seqs[i]``; outcome in ``cache.status``."""
    c = _cache(cache)
    a = _list(c, "seqs", seqs)
    b = _list(c, "counts", counts, seqs.shape[0])
    _launch(c, stream, lib().bdlm_cache_grow, c._ref, seqs.shape[0], a, b)


def cache_fork(cache: Cache, parents, children, stream=None):
    """Sequences ``children[i]`` become copies of ``parents[i]`` that share full pages; outcome in ``cache.status``."""
    c = _cache(cache)
    a = _list(c, "parents", parents)
    b = _list(c, "children", children, parents.shape[0])
    _launch(c, stream, lib().bdlm_cache_fork, c._ref, parents.shape[0], a, b)


def cache_free(cache: Cache, seqs, stream=None):
    """Empties sequences and gives back the pages that no other sequence holds."""
    c = _cache(cache)
    a = _list(c, "seqs", seqs)
    _launch(c, stream, lib().bdlm_cache_free, c._ref, seqs.shape[0], a)


def cache_compact(cache: Cache, stream=None):
    """Moves live pages into the holes below them, so that the free pages are the last ones."""
    c = _cache(cache)
    _launch(c, stream, lib().bdlm_cache_compact, c._ref)


def cache_write(cache: Cache, layer: int, seqs, counts, k, v, starts: Optional[torch.Tensor] = None, stream=None):
    """K and V rows ``[rows][kv_heads][head_dim]`` of the last ``counts[i]`` tokens of the sequences, in one layer: from
    row ``starts[i]`` on, or, without ``starts``, an equal share of the rows each (of which the first ``counts[i]``)."""
    c = _cache(cache)
    a = _list(c, "seqs", seqs)
    n = seqs.shape[0]
    b = _list(c, "counts", counts, n)
    at = _list(c, "starts", starts, n) if starts is not None else None
    rk, rv = _rows(c, "k", k, c.kv_heads, 0), _rows(c, "v", v, c.kv_heads, 0)
    rows = k.shape[0]
    if rows != v.shape[0]:
        raise ValueError(f"k has {rows} rows, v has {v.shape[0]}")
    _launch(c, stream, lib().bdlm_cache_write, c._ref, _int("layer", layer), n, a, b, at, rows, rk, rv)


def _check_q(c, q):
    if not isinstance(q, torch.Tensor) or q.dim() != 4:
        raise ValueError("q must be a [requests][rows][heads][head_dim] tensor")
    R, n, H, D = q.shape
    _expect("q", q, c.dtype, (R, n, H, c.head_dim))
    if q.get_device() != c.gpu:
        raise ValueError(f"q must be on {c.device}, got {q.device}")
    return R, n, H


def _new_outputs(q):
    R, n, H, _ = q.shape
    return torch.empty_like(q), q.new_empty((R, H, n), dtype=torch.float32)


def prefix_attn_workspace_bytes(q, cache: Cache, prefix: int = 0) -> int:
    """Workspace of :func:`prefix_attn` for queries like ``q``."""
    c = _cache(cache)
    R, n, H = _check_q(c, q)
    return int(lib().bdlm_prefix_attn_workspace_bytes(c._ref, R, n, H, _int("prefix", prefix)))


def prefix_attn(q, cache: Cache, layer: int, seqs, prefix: int = 0, block: bool = False, scale: float = 0.0,
                out: Optional[tuple] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of the last ``rows`` tokens of the sequences ``seqs`` (int32 ``[requests]``) over their keys in the
    cache: q ``[requests][rows][heads][head_dim]``, causal, or, with ``block``, every row sees all of its sequence.
    The first ``prefix`` tokens, the same in all requests, may be read once for all of them, through the table of the
    first one, which has to hold them all.
    Returns ``(o, lse)`` with ``lse [requests][heads][rows]`` fp32, or writes into ``out``.  ``workspace``: a device
    tensor of :func:`prefix_attn_workspace_bytes` (calls that may overlap in time need one each); allocated if not
    given."""
    c = _cache(cache)
    R, n, H = _check_q(c, q)
    a = _list(c, "seqs", seqs, R)
    layer, prefix = _int("layer", layer), _int("prefix", prefix)
    if out is None:
        o, lse = _made(stream, c.device, _new_outputs, q)
    else:
        if len(out) != 2:
            raise ValueError("out must be (o, lse)")
        o, lse = out
        _expect("o", o, c.dtype, q.shape)
        _expect("lse", lse, torch.float32, (R, H, n))
        if o.get_device() != c.gpu or lse.get_device() != c.gpu:
            raise ValueError(f"o and lse must be on {c.device}")
    if workspace is None:
        nbytes = lib().bdlm_prefix_attn_workspace_bytes(c._ref, R, n, H, prefix)
        workspace = _workspace(None, nbytes, c.device, stream)
    else:
        _workspace(workspace, 0, c.device, stream)
        nbytes = workspace.numel() * workspace.element_size()
    _launch(c, stream, lib().bdlm_prefix_attn, c._ref, layer, R, a, n, H, prefix, 1 if block else 0, scale,
            q.data_ptr(), o.data_ptr(), lse.data_ptr(), workspace.data_ptr(), nbytes)
    return o, lse
