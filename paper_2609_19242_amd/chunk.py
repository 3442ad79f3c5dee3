"""Attention of chunks of new tokens over a paged cache: requests with different numbers of rows in one call, one for a
decoding request, many for a piece of a prompt.

A :class:`ChunkPlan` (:func:`chunk_plan`) is made on the device once for a step and serves every layer
(:func:`chunk_attn`).  The rules and layouts are those of ``bdlm_chunk_plan`` and ``bdlm_chunk_attn`` in
``include/bdlm_attn.h``.  With ``stream``, a call runs there and is not ordered against the current stream, as in the
cache's operations.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from . import _launch, _made, _raw_stream, _stream, _torch_stream, lib
from .cache import _cache, _Cache, _list
from .packed import _as_long, _int, _lse, _Rows, _workspace

__all__ = ["ChunkPlan", "chunk_plan", "chunk_attn", "chunk_attn_workspace_bytes"]

STARTS = 64  # BDLM_CHUNK_STARTS


class _Chunk(ctypes.Structure):  # bdlm_chunk
    _fields_ = [(n, ctypes.c_int64) for n in ("requests", "rows", "block_size", "window")] + \
               [("heads", ctypes.c_int32), ("sinks", ctypes.c_int32), ("scale", ctypes.c_float), ("reserved", ctypes.c_int32)]


def declare(L: ctypes.CDLL):
    vp, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
    head = [ctypes.POINTER(_Cache), ctypes.POINTER(_Chunk)]
    for name in ("bdlm_chunk_plan_bytes", "bdlm_chunk_workspace_bytes"):
        getattr(L, name).argtypes = head
        getattr(L, name).restype = sz
    L.bdlm_chunk_plan.argtypes = head + [vp, vp, vp, sz, vp]
    L.bdlm_chunk_attn.argtypes = head + [i64, vp, sz, _Rows, _Rows, vp, i64, i32, vp, sz, vp]
    for name in ("bdlm_chunk_plan", "bdlm_chunk_attn"):
        getattr(L, name).restype = ctypes.c_int


class ChunkPlan:
    """The work of a step of attention over ``cache`` (see :func:`chunk_plan`).  ``starts``: the requests' first rows,
    int32 ``[requests]``, as :func:`cache_write` takes them."""

    def __init__(self, cache, record: _Chunk, items: torch.Tensor, stream):
        self.cache, self._record, self._items, self._workspace_bytes = cache, record, items, None
        self._ref, self._at, self._bytes = ctypes.byref(record), items.data_ptr(), items.numel() * 4
        self.requests, self.rows, self.heads = record.requests, record.rows, record.heads
        self.dtype, self.device, self.gpu, self.head_dim = cache.dtype, cache.device, cache.gpu, cache.head_dim
        # (the items come from the memory of the stream that makes them)
        self._tensors, self._streams = (items,), set()
        if self.gpu >= 0:  # (its own GPU's, which may not be the current one)
            self._streams.add(_raw_stream(self.gpu) if stream is None else _stream(stream))

    @property
    def workspace_bytes(self):
        if self._workspace_bytes is None:
            self._workspace_bytes = int(lib().bdlm_chunk_workspace_bytes(self.cache._ref, self._ref))
        return self._workspace_bytes

    @property
    def starts(self):
        return self._items[STARTS // 4:STARTS // 4 + self.requests]

    def __repr__(self):
        return f"ChunkPlan(requests={self.requests}, rows={self.rows}, heads={self.heads}, {self.cache!r})"


def _launch_plan(plan, stream, call, *args):
    """:func:`_launch`, of the plan's memory and the cache's."""
    _launch(plan, stream, call, *args)
    c = plan.cache
    for handle in plan._streams - c._streams:
        for t in c._tensors:
            t.record_stream(_torch_stream(handle, c.device))
        c._streams.add(handle)


def chunk_plan(cache, seqs, counts, rows: int, heads: int, block_size: int = 1, window: int = 0, sinks: int = 0,
               scale: float = 0.0, out: Optional[ChunkPlan] = None, stream=None) -> ChunkPlan:
    """The plan of a step in which sequence ``seqs[r]`` of ``cache`` has ``counts[r]`` new tokens (int32 lists on the
    GPU; after :func:`cache_grow`): their query rows lie one after the other in tensors of ``rows`` rows of ``heads``
    heads.  Each row sees the keys up to the end of its block of ``block_size`` tokens (1: up to itself), with
    ``window`` only the last ``window`` of those and its sequence's first ``sinks`` tokens.  ``out``: an earlier plan of
    the same cache, requests, rows and heads, which is overwritten (in a graph, say).  A captured :func:`chunk_attn`
    keeps the block size, window and sinks that its plan had then: replayed with another plan in the same place, it
    makes all rows NaN."""
    c = _cache(cache)
    a = _list(c, "seqs", seqs)
    n = seqs.shape[0]
    b = _list(c, "counts", counts, n)
    if not math.isfinite(scale):
        raise ValueError("scale is not finite")
    rec = _Chunk(n, _int("rows", rows), _int("block_size", block_size), _int("window", window), _int("heads", heads, 32),
                 _int("sinks", sinks, 32), scale, 0)
    ref = ctypes.byref(rec)
    nbytes = lib().bdlm_chunk_plan_bytes(c._ref, ref)
    if out is None:
        # (0: refused, by the call below)
        items, = _made(stream, c.device, lambda: (torch.empty(max(64, nbytes // 4), dtype=torch.int32, device=c.device),))
        plan = ChunkPlan(c, rec, items, stream)
    else:
        if not isinstance(out, ChunkPlan):
            raise TypeError(f"out must be a ChunkPlan, got {type(out).__name__}")
        if out.cache is not c or (out.requests, out.rows, out.heads) != (n, rec.rows, rec.heads):
            raise ValueError("out must be a plan of the same cache, requests, rows and heads")
        plan = out
    _launch_plan(plan, stream, lib().bdlm_chunk_plan, c._ref, ref, a, b, plan._at, plan._bytes)
    if out is not None:
        ctypes.memmove(ctypes.byref(plan._record), ref, ctypes.sizeof(rec))
        plan._workspace_bytes = None
    return plan


def _check_plan(plan):
    if not isinstance(plan, ChunkPlan):
        raise TypeError(f"plan must be a ChunkPlan, got {type(plan).__name__}")


def chunk_attn_workspace_bytes(plan: ChunkPlan) -> int:
    """Workspace of :func:`chunk_attn`."""
    _check_plan(plan)
    return plan.workspace_bytes


def _new_outputs(plan):
    return (torch.empty(plan.rows, plan.heads, plan.head_dim, dtype=plan.dtype, device=plan.device),
            torch.empty(plan.heads, plan.rows, dtype=torch.float32, device=plan.device))


def chunk_attn(plan: ChunkPlan, q, layer: int, out: Optional[tuple] = None, workspace: Optional[torch.Tensor] = None,
               stream=None):
    """Attention of the plan's rows over their sequences' keys in ``layer`` of the cache: q ``[rows][heads][head_dim]``
    (rows may lie apart, as in a fused projection).  Returns ``(o, lse)`` with ``lse [heads][rows]`` fp32, or writes
    into ``out``; rows behind the last request's are left as they are there, and are 0 (lse: -inf) in new outputs.
    ``workspace``: a device tensor of :func:`chunk_attn_workspace_bytes` (calls that may overlap in time need one each);
    allocated if not given."""
    _check_plan(plan)
    H, n = plan.heads, plan.rows
    rq = _as_long(plan, "q", q, H, n)
    layer = _int("layer", layer)
    if out is None:
        o, lse = _made(stream, plan.device, _new_outputs, plan)
        ro = _Rows(o.data_ptr(), H * plan.head_dim)
    else:
        if len(out) != 2:
            raise ValueError("out must be (o, lse)")
        o, lse = out
        ro = _as_long(plan, "o", o, H, n)
        _lse(plan, lse, n)
    at, nbytes = None, plan.workspace_bytes
    if workspace is not None or nbytes > 0:
        workspace = _workspace(workspace, nbytes, plan.device, stream)
        at, nbytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _launch_plan(plan, stream, lib().bdlm_chunk_attn, plan.cache._ref, plan._ref, layer, plan._at, plan._bytes, rq, ro,
                 lse.data_ptr(), n, 1 if out is None else 0, at, nbytes)
    return o, lse
