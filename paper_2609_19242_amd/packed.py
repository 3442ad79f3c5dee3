"""Packed attention: prompts and training texts of different lengths in one call.

A :class:`PackedPlan` (:func:`packed_plan`) is made once for a set of sequence lengths and serves every layer,
forward (:func:`packed_fwd`) and backward (:func:`packed_bwd`).  The rules and layouts are those of
``bdlm_packed_fwd`` in ``include/bdlm_attn.h``.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import _check, _dtype_code, _expect, _on_device, _torch_stream, device_stream, lib

__all__ = ["PackedPlan", "packed_plan", "packed_fwd", "packed_bwd"]


class _Packed(ctypes.Structure):  # bdlm_packed
    _fields_ = [("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("scale", ctypes.c_float), ("reserved", ctypes.c_int32),
                ("block_size", ctypes.c_int64), ("window", ctypes.c_int64)]


class _Seq(ctypes.Structure):  # bdlm_packed_seq
    _fields_ = [("q_start", ctypes.c_int64), ("q_len", ctypes.c_int64),
                ("k_start", ctypes.c_int64), ("k_len", ctypes.c_int64)]


class _Plan(ctypes.Structure):  # bdlm_packed_plan
    _fields_ = [("problem", _Packed), ("q_rows", ctypes.c_int64), ("k_rows", ctypes.c_int64),
                ("q_items", ctypes.c_int32), ("k_items", ctypes.c_int32), ("n_sums", ctypes.c_int32),
                ("slots", ctypes.c_int32), ("teams", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("bytes", ctypes.c_size_t), ("workspace_bytes", ctypes.c_size_t)]


class _Rows(ctypes.Structure):  # bdlm_rows
    _fields_ = [("ptr", ctypes.c_void_p), ("stride", ctypes.c_int64)]


def declare(L: ctypes.CDLL):
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    L.bdlm_packed_plan_make.argtypes = [ctypes.POINTER(_Packed), ctypes.c_int64, ctypes.POINTER(_Seq), vp, sz,
                                        ctypes.POINTER(_Plan)]
    L.bdlm_packed_fwd.argtypes = [ctypes.POINTER(_Plan), vp] + [_Rows] * 4 + [vp, ctypes.c_int64, vp]
    L.bdlm_packed_bwd.argtypes = [ctypes.POINTER(_Plan), vp] + [_Rows] * 4 + [vp, ctypes.c_int64] + [_Rows] * 4 + \
        [vp, sz, vp]
    for name in ("bdlm_packed_plan_make", "bdlm_packed_fwd", "bdlm_packed_bwd"):
        getattr(L, name).restype = ctypes.c_int


class PackedPlan:
    """The work items of packed calls over some sequences, on ``device`` (see :func:`packed_plan`)."""

    def __init__(self, record: _Plan, items: torch.Tensor, dtype: torch.dtype):
        self._record, self._items, self.dtype = record, items, dtype
        p = record.problem
        self.heads, self.kv_heads, self.head_dim = p.heads, p.kv_heads, p.head_dim
        self.q_rows, self.k_rows = record.q_rows, record.k_rows
        self.workspace_bytes = record.workspace_bytes
        self.device = items.device

    def __repr__(self):
        return (f"PackedPlan(q_rows={self.q_rows}, k_rows={self.k_rows}, heads={self.heads}, kv_heads={self.kv_heads}, "
                f"head_dim={self.head_dim}, {self.dtype}, {self.device})")


def _ints(name, xs, n=None):
    if isinstance(xs, torch.Tensor):
        if xs.is_cuda or xs.dim() != 1 or xs.dtype not in (torch.int32, torch.int64):
            raise ValueError(f"{name} must be a one-dimensional integer tensor on the CPU, or a sequence of ints")
        xs = xs.tolist()
    xs = [int(x) for x in xs]
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
    p = _Packed(heads, kv_heads, head_dim, _dtype_code(dtype), scale, 0, block_size, window)
    seqs = (_Seq * max(1, n))(*[_Seq(a, b, c, d) for a, b, c, d in zip(qs, ql, ks, kl)])
    rec = _Plan()
    _check(lib().bdlm_packed_plan_make(ctypes.byref(p), n, seqs, None, 0, ctypes.byref(rec)))
    host = torch.empty(max(16, rec.bytes), dtype=torch.uint8)
    _check(lib().bdlm_packed_plan_make(ctypes.byref(p), n, seqs, host.data_ptr(), host.numel(), ctypes.byref(rec)))
    return PackedPlan(rec, host.to(device), dtype)


def _rows(plan, name, t, heads, at_least):
    """A ``[rows][heads][head_dim]`` tensor whose rows may lie further apart than they are long."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor, got {type(t).__name__}")
    if t.dtype != plan.dtype:
        raise TypeError(f"{name} must be {plan.dtype}, got {t.dtype}")
    D = plan.head_dim
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != D:
        raise ValueError(f"{name} must have shape (rows, {heads}, {D}), got {tuple(t.shape)}")
    n, st = t.shape[0], t.stride()
    if n < at_least:
        raise ValueError(f"{name} has {n} rows, the plan's sequences end at row {at_least}")
    if n and (st[2] != 1 or (heads > 1 and st[1] != D) or (n > 1 and st[0] < heads * D)):
        raise ValueError(f"{name} must hold each row's heads contiguously (only rows may lie apart)")
    return _Rows(t.data_ptr(), st[0] if n > 1 else heads * D)


def _check_plan(plan):
    if not isinstance(plan, PackedPlan):
        raise TypeError(f"plan must be a PackedPlan, got {type(plan).__name__}")


def _like(t, rows, heads, D):
    return torch.empty((rows, heads, D), dtype=t.dtype, device=t.device)


def packed_fwd(plan: PackedPlan, q, k, v, out: Optional[tuple] = None, stream=None):
    """Attention of the plan's sequences: q ``[rows][heads][D]``, k and v ``[rows][kv_heads][D]`` (rows may lie apart,
    as in a fused projection).  Returns ``(o, lse)`` with ``lse [heads][rows]`` fp32, or writes into ``out``; rows of
    no sequence are left as they are (in new outputs: undefined)."""
    _check_plan(plan)
    H, KV, D = plan.heads, plan.kv_heads, plan.head_dim
    rq, rk, rv = (_rows(plan, *a) for a in (("q", q, H, plan.q_rows), ("k", k, KV, plan.k_rows),
                                            ("v", v, KV, plan.k_rows)))
    n = q.shape[0]
    if out is not None:
        if len(out) != 2:
            raise ValueError("out must be (o, lse)")
        o, lse = out
        _rows(plan, "o", o, H, n)
        if o.shape[0] != n:
            raise ValueError(f"o must have as many rows as q ({n}), got {o.shape[0]}")
        _expect("lse", lse, torch.float32, (H, n))
    _on_device(plan.device, q=q, k=k, v=v)
    if out is None:
        o, lse = _like(q, n, H, D), torch.empty((H, n), dtype=torch.float32, device=q.device)
    else:
        _on_device(plan.device, o=o, lse=lse)
    ro = _rows(plan, "o", o, H, plan.q_rows)
    with device_stream(plan.device, stream) as s:
        _check(lib().bdlm_packed_fwd(ctypes.byref(plan._record), plan._items.data_ptr(), rq, rk, rv, ro,
                                     lse.data_ptr(), n, s))
    return o, lse


def packed_bwd(plan: PackedPlan, q, k, v, o, lse, do, out: Optional[tuple] = None,
               workspace: Optional[torch.Tensor] = None, stream=None):
    """Backward of :func:`packed_fwd`; returns ``(dq, dk, dv)``, or writes into ``out``.  ``workspace``: a device
    tensor of ``plan.workspace_bytes`` bytes (calls that may overlap in time need one each); allocated if not given."""
    _check_plan(plan)
    H, KV, D = plan.heads, plan.kv_heads, plan.head_dim
    n, nk = (t.shape[0] if isinstance(t, torch.Tensor) and t.dim() else 0 for t in (q, k))
    ins = [("q", q, H, plan.q_rows), ("k", k, KV, plan.k_rows), ("v", v, KV, plan.k_rows), ("o", o, H, n),
           ("do", do, H, n)]
    rq, rk, rv, ro, rdo = (_rows(plan, *a) for a in ins)
    for name, t in (("o", o), ("do", do)):
        if t.shape[0] != n:
            raise ValueError(f"{name} must have as many rows as q ({n}), got {t.shape[0]}")
    _expect("lse", lse, torch.float32, (H, n))
    if out is not None:
        if len(out) != 3:
            raise ValueError("out must be (dq, dk, dv)")
        for name, t, h, m in (("dq", out[0], H, n), ("dk", out[1], KV, nk), ("dv", out[2], KV, v.shape[0])):
            _rows(plan, name, t, h, m)
    _on_device(plan.device, q=q, k=k, v=v, o=o, lse=lse, do=do)
    if out is None:
        out = _like(q, n, H, D), _like(k, nk, KV, D), _like(v, v.shape[0], KV, D)
    else:
        _on_device(plan.device, dq=out[0], dk=out[1], dv=out[2])
    dq, dk, dv = out
    outs = [_rows(plan, "dq", dq, H, plan.q_rows), _rows(plan, "dk", dk, KV, plan.k_rows),
            _rows(plan, "dv", dv, KV, plan.k_rows)]
    workspace = _workspace(workspace, plan.workspace_bytes, plan.device, stream)
    with device_stream(plan.device, stream) as s:
        _check(lib().bdlm_packed_bwd(ctypes.byref(plan._record), plan._items.data_ptr(), rq, rk, rv, ro,
                                     lse.data_ptr(), n, rdo, *outs, workspace.data_ptr(),
                                     workspace.numel() * workspace.element_size(), s))
    return dq, dk, dv


def _workspace(workspace, nbytes, device, stream):
    if workspace is not None:
        if not isinstance(workspace, torch.Tensor) or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor")
        _on_device(device, workspace=workspace)
        return workspace
    workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
    if stream is not None:  # used on that stream after this call has dropped it
        workspace.record_stream(_torch_stream(stream, device))
    return workspace
