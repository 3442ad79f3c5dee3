"""Packed attention: prompts and training texts of different lengths in one call.

A :class:`PackedPlan` (:func:`packed_plan`) is made once for a set of sequence lengths and serves every layer,
forward (:func:`packed_fwd`) and backward (:func:`packed_bwd`).  The rules and layouts are those of
``bdlm_packed_fwd`` in ``include/bdlm_attn.h``.  With ``stream``, a call runs there and is not ordered against the
current stream: the caller orders what it reads before it, keeps that until it has run, and orders what uses its results
behind it.
"""
from __future__ import annotations

import ctypes
import math
import operator
from typing import Optional, Sequence

import torch

from . import _check, _dtype_code, _expect, _launch, _made, _memory_of, _on_device, lib

__all__ = ["PackedPlan", "packed_plan", "packed_fwd", "packed_bwd"]


class _Packed(ctypes.Structure):  # bdlm_packed
    _fields_ = [("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("scale", ctypes.c_float), ("reserved", ctypes.c_int32),
                ("block_size", ctypes.c_int64), ("window", ctypes.c_int64)]


class _Seq(ctypes.Structure):  # bdlm_packed_seq
    _fields_ = [("q_start", ctypes.c_int64), ("q_len", ctypes.c_int64),
                ("k_start", ctypes.c_int64), ("k_len", ctypes.c_int64)]


class _Chunks(ctypes.Structure):  # bdlm_packed_chunks
    _fields_ = [(n, ctypes.c_int32) for n in ("items", "sums", "slots", "reserved")]


class _Plan(ctypes.Structure):  # bdlm_packed_plan
    _fields_ = [("problem", _Packed), ("q_rows", ctypes.c_int64), ("k_rows", ctypes.c_int64),
                ("q_items", ctypes.c_int32), ("k_items", ctypes.c_int32), ("n_sums", ctypes.c_int32),
                ("slots", ctypes.c_int32), ("teams", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("fwd", _Chunks), ("dq", _Chunks),
                ("bytes", ctypes.c_size_t), ("workspace_bytes", ctypes.c_size_t), ("fwd_workspace_bytes", ctypes.c_size_t)]


class _Rows(ctypes.Structure):  # bdlm_rows
    _fields_ = [("ptr", ctypes.c_void_p), ("stride", ctypes.c_int64)]


def declare(L: ctypes.CDLL):
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    L.bdlm_packed_plan_make.argtypes = [ctypes.POINTER(_Packed), ctypes.c_int64, ctypes.POINTER(_Seq), vp, sz,
                                        ctypes.POINTER(_Plan)]
    L.bdlm_packed_fwd.argtypes = [ctypes.POINTER(_Plan), vp] + [_Rows] * 4 + [vp, ctypes.c_int64, vp, sz, vp]
    L.bdlm_packed_bwd.argtypes = [ctypes.POINTER(_Plan), vp] + [_Rows] * 4 + [vp, ctypes.c_int64] + [_Rows] * 4 + \
        [vp, sz, vp]
    for name in ("bdlm_packed_plan_make", "bdlm_packed_fwd", "bdlm_packed_bwd"):
        getattr(L, name).restype = ctypes.c_int


class PackedPlan:
    """The work items of packed calls over some sequences, on ``device`` (see :func:`packed_plan`)."""

    def __init__(self, record: _Plan, items: torch.Tensor, dtype: torch.dtype, held=(0, 0)):
        self._record, self._items, self.dtype = record, items, dtype
        self._held = held  # query and key rows that belong to a sequence
        self._tensors, self._streams = (items,), set()
        self._ref, self._at = ctypes.byref(record), items.data_ptr()
        p = record.problem
        self.heads, self.kv_heads, self.head_dim = p.heads, p.kv_heads, p.head_dim
        self.q_rows, self.k_rows = record.q_rows, record.k_rows
        self.workspace_bytes, self.fwd_workspace_bytes = record.workspace_bytes, record.fwd_workspace_bytes
        self.device, self.gpu = items.device, items.get_device()  # (gpu: -1 on the CPU)

    def __repr__(self):
        return (f"PackedPlan(q_rows={self.q_rows}, k_rows={self.k_rows}, heads={self.heads}, kv_heads={self.kv_heads}, "
                f"head_dim={self.head_dim}, {self.dtype}, {self.device})")


def _int(name, x, bits=64):
    """``x`` as the C ABI's integer (which would take the low bits of a larger one)."""
    x = operator.index(x)
    if not -1 << bits - 1 <= x < 1 << bits - 1:
        raise ValueError(f"{name} {x} does not fit {bits} bits")
    return x


def _ints(name, xs, n=None):
    if isinstance(xs, torch.Tensor):
        if xs.is_cuda or xs.dim() != 1 or xs.dtype not in (torch.int32, torch.int64):
            raise ValueError(f"{name} must be a one-dimensional integer tensor on the CPU, or a sequence of ints")
        xs = xs.tolist()
    xs = [operator.index(x) for x in xs]
    if xs:
        _int(name, min(xs)), _int(name, max(xs))
    if n is not None and len(xs) != n:
        raise ValueError(f"{name} has {len(xs)} entries for {n} sequences")
    return xs


def packed_plan(q_lens: Sequence[int], k_lens: Optional[Sequence[int]] = None, *, heads: int, kv_heads: int,
                head_dim: int, dtype, block_size: int = 1, window: int = 0, scale: float = 0.0,
                q_starts: Optional[Sequence[int]] = None, k_starts: Optional[Sequence[int]] = None,
                device="cuda") -> PackedPlan:
    """The plan of packed calls over sequences of ``q_lens`` query rows and ``k_lens`` keys (default: the same).

    A sequence's queries are its last ``q_len`` tokens; each sees the keys up to the end of its block of
    ``block_size`` tokens (1: up to itself), with ``window`` only the last ``window`` of those.  Sequences lie one
    after the other, or at the rows ``q_starts`` / ``k_starts`` (a padded batch, say): in order, without overlap.
    The lengths are host values; the plan's items are copied to ``device`` (not while a graph is captured)."""
    ql = _ints("q_lens", q_lens)
    n = len(ql)
    kl = ql if k_lens is None else _ints("k_lens", k_lens, n)

    def starts(name, given, lens):
        if given is not None:
            return _ints(name, given, n)
        out, at = [], 0
        for x in lens:
            out.append(at)
            at += x
        return out

    qs = starts("q_starts", q_starts, ql)
    ks = starts("k_starts", k_starts, kl) if k_starts is not None or k_lens is not None or q_starts is None else qs
    p = _Packed(_int("heads", heads, 32), _int("kv_heads", kv_heads, 32), _int("head_dim", head_dim, 32), _dtype_code(dtype),
                scale, 0, _int("block_size", block_size), _int("window", window))
    seqs = (_Seq * max(1, n))(*[_Seq(a, b, c, d) for a, b, c, d in zip(qs, ql, ks, kl)])
    rec = _Plan()
    _check(lib().bdlm_packed_plan_make(ctypes.byref(p), n, seqs, None, 0, ctypes.byref(rec)))
    host = torch.empty(max(16, rec.bytes), dtype=torch.uint8)
    _check(lib().bdlm_packed_plan_make(ctypes.byref(p), n, seqs, host.data_ptr(), host.numel(), ctypes.byref(rec)))
    return PackedPlan(rec, host.to(device), dtype, (sum(ql), sum(kl)))


def _rows(like, name, t, heads, at_least):
    """A ``[rows][heads][head_dim]`` tensor whose rows may lie further apart than they are long, in the dtype and on the
    device of ``like`` (a plan or a cache)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor, got {type(t).__name__}")
    if t.dtype is not like.dtype:
        raise TypeError(f"{name} must be {like.dtype}, got {t.dtype}")
    D, shape, st = like.head_dim, t.shape, t.stride()
    if len(shape) != 3 or shape[1] != heads or shape[2] != D:
        raise ValueError(f"{name} must have shape (rows, {heads}, {D}), got {tuple(shape)}")
    n, s0 = shape[0], st[0]
    if n < at_least:
        raise ValueError(f"{name} has {n} rows, {at_least} are needed")
    if n <= 1:
        s0 = heads * D
    if n and (st[2] != 1 or (heads > 1 and st[1] != D) or s0 < heads * D):
        raise ValueError(f"{name} must hold each row's heads contiguously (only rows may lie apart)")
    if t.get_device() != like.gpu:
        raise ValueError(f"{name} must be on {like.device}, got {t.device}")
    return _Rows(t.data_ptr(), s0)


def _check_plan(plan):
    if not isinstance(plan, PackedPlan):
        raise TypeError(f"plan must be a PackedPlan, got {type(plan).__name__}")


# New outputs, filled where a call does not write all of them.
def _fwd_outputs(plan, q):
    n, H = q.shape[0], plan.heads
    o, lse = q.new_empty((n, H, plan.head_dim)), q.new_empty((H, n), dtype=torch.float32)
    return (o, lse) if n == plan._held[0] else (o.zero_(), lse.fill_(-math.inf))


def _bwd_outputs(plan, q, k, v):
    n, nk, nv, H, KV, D = q.shape[0], k.shape[0], v.shape[0], plan.heads, plan.kv_heads, plan.head_dim
    hq, hk = plan._held
    dq, dk, dv = q.new_empty((n, H, D)), k.new_empty((nk, KV, D)), v.new_empty((nv, KV, D))
    return (dq if n == hq else dq.zero_(), dk if nk == hk else dk.zero_(), dv if nv == hk else dv.zero_())


def packed_fwd(plan: PackedPlan, q, k, v, out: Optional[tuple] = None, workspace: Optional[torch.Tensor] = None,
               stream=None):
    """Attention of the plan's sequences: q ``[rows][heads][D]``, k and v ``[rows][kv_heads][D]`` (rows may lie apart,
    as in a fused projection).  Returns ``(o, lse)`` with ``lse [heads][rows]`` fp32, or writes into ``out``; rows of
    no sequence are left as they are there, and are 0 (lse: -inf) in new outputs.  ``workspace``: a device tensor of
    ``plan.fwd_workspace_bytes`` bytes, if that is not 0 (as in :func:`packed_bwd`)."""
    _check_plan(plan)
    H, KV = plan.heads, plan.kv_heads
    rq, rk, rv = (_rows(plan, "q", q, H, plan.q_rows), _rows(plan, "k", k, KV, plan.k_rows),
                  _rows(plan, "v", v, KV, plan.k_rows))
    n = q.shape[0]
    if out is None:
        o, lse = _made(stream, plan.device, _fwd_outputs, plan, q)
        ro = _Rows(o.data_ptr(), H * plan.head_dim)
    else:
        if len(out) != 2:
            raise ValueError("out must be (o, lse)")
        o, lse = out
        ro = _as_long(plan, "o", o, H, n)
        _lse(plan, lse, n)
    at = nbytes = 0
    if plan.fwd_workspace_bytes:
        workspace = _workspace(workspace, plan.fwd_workspace_bytes, plan.device, stream)
        at, nbytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _launch(plan, stream, lib().bdlm_packed_fwd, plan._ref, plan._at, rq, rk, rv, ro, lse.data_ptr(), n, at, nbytes)
    return o, lse


def packed_bwd(plan: PackedPlan, q, k, v, o, lse, do, out: Optional[tuple] = None,
               workspace: Optional[torch.Tensor] = None, stream=None):
    """Backward of :func:`packed_fwd`; returns ``(dq, dk, dv)``, or writes into ``out``; rows of no sequence are left as
    they are there, and are 0 in new outputs.  ``workspace``: a device tensor of ``plan.workspace_bytes`` bytes (calls
    that may overlap in time need one each); allocated if not given."""
    _check_plan(plan)
    H, KV, D = plan.heads, plan.kv_heads, plan.head_dim
    rq, rk, rv = (_rows(plan, "q", q, H, plan.q_rows), _rows(plan, "k", k, KV, plan.k_rows),
                  _rows(plan, "v", v, KV, plan.k_rows))
    n, nk, nv = q.shape[0], k.shape[0], v.shape[0]
    ro, rdo = _as_long(plan, "o", o, H, n), _as_long(plan, "do", do, H, n)
    _lse(plan, lse, n)
    if out is None:
        dq, dk, dv = _made(stream, plan.device, _bwd_outputs, plan, q, k, v)
        outs = _Rows(dq.data_ptr(), H * D), _Rows(dk.data_ptr(), KV * D), _Rows(dv.data_ptr(), KV * D)
    else:
        if len(out) != 3:
            raise ValueError("out must be (dq, dk, dv)")
        dq, dk, dv = out
        outs = _as_long(plan, "dq", dq, H, n), _as_long(plan, "dk", dk, KV, nk), _as_long(plan, "dv", dv, KV, nv)
    workspace = _workspace(workspace, plan.workspace_bytes, plan.device, stream)
    _launch(plan, stream, lib().bdlm_packed_bwd, plan._ref, plan._at, rq, rk, rv, ro, lse.data_ptr(), n, rdo,
            *outs, workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return dq, dk, dv


def _as_long(plan, name, t, heads, n):
    r = _rows(plan, name, t, heads, n)
    if t.shape[0] != n:
        raise ValueError(f"{name} must have {n} rows, got {t.shape[0]}")
    return r


def _lse(plan, lse, n):
    _expect("lse", lse, torch.float32, (plan.heads, n))
    if lse.get_device() != plan.gpu:
        raise ValueError(f"lse must be on {plan.device}, got {lse.device}")


def _workspace(workspace, nbytes, device, stream):
    if workspace is not None:
        if not isinstance(workspace, torch.Tensor) or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor")
        _on_device(device, workspace=workspace)
        return workspace
    if stream is None:
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
    with _memory_of(stream, device):
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
