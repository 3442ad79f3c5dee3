"""Norms of queries and keys for each head with the position rotation, in one pass: what comes between the projections
and any of the attention calls.

A :class:`Rotary` (:func:`rotary`) says how heads turn; it is made once for a model and knows no device.
:func:`qk_rotate_fwd` and :func:`qk_rotate_bwd` have the rules and layouts of ``bdlm_qk_rotate_fwd`` and ``_bwd`` in
``include/bdlm_attn.h``.  With ``stream``, a call runs there and is not ordered against the current stream, as in packed
calls.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Sequence

import torch

from . import _dtype_code, _expect, _launch, _made, lib
from .packed import _as_long, _int, _Rows, _rows, _workspace

__all__ = ["Rotary", "rotary", "qk_rotate_fwd", "qk_rotate_bwd"]

MAX_AXES = 4  # BDLM_MAX_AXES


class _Rotary(ctypes.Structure):  # bdlm_rotary
    _fields_ = [(n, ctypes.c_int32) for n in ("head_dim", "dim", "interleaved", "axes")] + \
               [("freq", ctypes.c_double * 64), ("axis", ctypes.c_int32 * 64)]


def declare(L: ctypes.CDLL):
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    head = [ctypes.POINTER(_Rotary), i32, i64, vp, i32, i32, _Rows, _Rows, vp, vp, ctypes.c_double]
    L.bdlm_qk_rotate_fwd.argtypes = head + [_Rows, _Rows, vp]
    L.bdlm_qk_rotate_bwd.argtypes = head + [_Rows] * 4 + [vp, vp, vp, sz, vp]
    L.bdlm_qk_rotate_workspace_bytes.argtypes = [i32]
    L.bdlm_qk_rotate_workspace_bytes.restype = sz
    for name in ("bdlm_qk_rotate_fwd", "bdlm_qk_rotate_bwd"):
        getattr(L, name).restype = ctypes.c_int


class Rotary:
    """How the heads' rows turn with their positions (see :func:`rotary`)."""

    def __init__(self, record: _Rotary):
        self._record, self._ref = record, ctypes.byref(record)
        self.head_dim, self.dim, self.axes = record.head_dim, record.dim, record.axes
        self.interleaved = bool(record.interleaved)
        self._calls = {}

    @property
    def freqs(self):
        """Radians per position of each pair."""
        return list(self._record.freq[:self.dim // 2])

    @property
    def pair_axes(self):
        """The position axis of each pair."""
        return list(self._record.axis[:self.dim // 2])

    def __repr__(self):
        return (f"Rotary(head_dim={self.head_dim}, dim={self.dim}, axes={self.axes}, "
                f"{'neighbours' if self.interleaved else 'halves'})")


def rotary(head_dim: int, dim: Optional[int] = None, base: float = 10000.0, sections: Optional[Sequence[int]] = None,
           own_ladders: bool = False, freqs: Optional[Sequence[float]] = None, interleaved: bool = False) -> Rotary:
    """The rotation of heads of ``head_dim`` elements, of which the first ``dim`` (default: all) turn in pairs: elements
    i and i + dim / 2, or, ``interleaved``, 2 i and 2 i + 1.

    ``sections``: how many of the pairs, in order, follow each position axis (time, height, width, say; default: one
    axis).  Pair i turns by ``base ** (-i / pairs)`` radians per position; with ``own_ladders`` every axis's pairs have
    a ladder of their own, ``base ** (-j / section)`` for its j-th pair; or by ``freqs[i]``."""
    head_dim = _int("head_dim", head_dim, 32)
    dim = head_dim if dim is None else _int("dim", dim, 32)
    if head_dim not in (64, 128) or not 16 <= dim <= head_dim or dim % 16:
        raise ValueError(f"head_dim must be 64 or 128 and dim a multiple of 16 up to it, got {head_dim} and {dim}")
    n = dim // 2
    sections = [n] if sections is None else [_int("section", x, 32) for x in sections]
    if not 1 <= len(sections) <= MAX_AXES or min(sections) < 0 or sum(sections) != n:
        raise ValueError(f"sections must be 1 to {MAX_AXES} numbers of pairs that add up to {n}, got {sections}")
    axis = [a for a, m in enumerate(sections) for _ in range(m)]
    if freqs is None:
        if not (math.isfinite(base) and base > 0):
            raise ValueError(f"base must be finite and positive, got {base}")
        freqs = [float(base) ** (-j / m) for m in sections for j in range(m)] if own_ladders else \
            [float(base) ** (-i / n) for i in range(n)]
    freqs = [float(f) for f in freqs]
    if len(freqs) != n or not all(abs(f) <= 2.0 ** 20 for f in freqs):
        raise ValueError(f"freqs must be {n} numbers of at most 2^20 radians per position")
    pad = 64 - n
    return Rotary(_Rotary(head_dim, dim, int(bool(interleaved)), len(sections), (ctypes.c_double * 64)(*freqs, *[0.0] * pad),
                          (ctypes.c_int32 * 64)(*axis, *[0] * pad)))


class _Call:
    """The dtype and device of a call's tensors."""

    _tensors = ()

    def __init__(self, dtype, device, gpu, head_dim):
        self.code = _dtype_code(dtype)
        self.dtype, self.device, self.gpu, self.head_dim = dtype, device, gpu, head_dim
        self._streams, self.workspace_bytes = set(), None


def _call(rot, q):
    """Those of q (kept with the rotation: a small call's host time is its launch)."""
    if not isinstance(rot, Rotary):
        raise TypeError(f"rot must be a Rotary, got {type(rot).__name__}")
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError(f"q must be a [rows][heads][{rot.head_dim}] tensor")
    key = q.dtype, q.get_device()
    c = rot._calls.get(key)
    if c is None:
        c = rot._calls[key] = _Call(q.dtype, q.device, key[1], rot.head_dim)
    return c


def _at(c, name, t, dtype, shape):
    """The address of a contiguous tensor of the call."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == c.gpu:
        return t.data_ptr()
    _expect(name, t, dtype, shape)
    raise ValueError(f"{name} must be on {c.device}, got {t.device}")


def _inputs(rot, q, k, positions, q_weight, k_weight, eps):
    """The arguments that both directions share, and the call's numbers."""
    c = _call(rot, q)
    n, H, _ = q.shape
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError(f"k must be a [rows][kv_heads][{rot.head_dim}] tensor")
    KV = k.shape[1]
    rq, rk = _rows(c, "q", q, H, n), _as_long(c, "k", k, KV, n)
    if not isinstance(positions, torch.Tensor) or positions.dim() not in (1, 2):
        raise ValueError("positions must be a [rows] or [axes][rows] tensor")
    at = _at(c, "positions", positions, torch.int32, (n,) if rot.axes == 1 and positions.dim() == 1 else (rot.axes, n))
    if eps is None:
        if q_weight is not None or k_weight is not None:
            raise ValueError("a weight needs a norm (eps)")
        return c, n, H, KV, (rot._ref, c.code, n, at, H, KV, rq, rk, None, None, 0.0)
    if not 2.0 ** -100 <= eps <= 2.0 ** 100:
        raise ValueError(f"eps must be within [2^-100, 2^100], or None for no norm, got {eps}")
    one = (c.head_dim,)
    return c, n, H, KV, (rot._ref, c.code, n, at, H, KV, rq, rk,
                         None if q_weight is None else _at(c, "q_weight", q_weight, c.dtype, one),
                         None if k_weight is None else _at(c, "k_weight", k_weight, c.dtype, one), eps)


def _new_rows(q, k):
    return torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format)


def _out_rows(c, out, names, q, k, stream):
    """The two outputs, new ones or the caller's, and their records."""
    if out is None:
        a, b = _made(stream, c.device, _new_rows, q, k)
        return (a, b), (_Rows(a.data_ptr(), q.shape[1] * c.head_dim), _Rows(b.data_ptr(), k.shape[1] * c.head_dim))
    if len(out) != 2:
        raise ValueError(f"out must be ({', '.join(names)})")
    n = q.shape[0]
    return tuple(out), [_as_long(c, x, t, like.shape[1], n) for x, t, like in zip(names, out, (q, k))]


def qk_rotate_fwd(rot: Rotary, q, k, positions, q_weight=None, k_weight=None, eps: Optional[float] = None,
                  out: Optional[tuple] = None, stream=None):
    """Queries ``[rows][heads][D]`` and keys ``[rows][kv_heads][D]`` (rows may lie apart, as in a fused projection),
    each head's row normed (``eps``; None: not) and scaled by ``q_weight`` / ``k_weight`` ``[D]``, then turned by its
    row's int32 ``positions`` (``[rows]``, with several axes ``[axes][rows]``).  Returns ``(q, k)``, or writes into
    ``out``, which may be the inputs."""
    c, n, H, KV, args = _inputs(rot, q, k, positions, q_weight, k_weight, eps)
    out, rows = _out_rows(c, out, ("q_out", "k_out"), q, k, stream)
    _launch(c, stream, lib().bdlm_qk_rotate_fwd, *args, *rows)
    return out


def _new_weight_grads(*weights):
    return [torch.empty_like(w, dtype=torch.float32) for w in weights]


def qk_rotate_bwd(rot: Rotary, q, k, positions, dq_out, dk_out, q_weight=None, k_weight=None,
                  eps: Optional[float] = None, out: Optional[tuple] = None, workspace: Optional[torch.Tensor] = None,
                  stream=None):
    """Backward of :func:`qk_rotate_fwd` from its inputs and its outputs' gradients.  Returns ``(dq, dk, dq_weight,
    dk_weight)``; the weights' gradients are fp32 (None without the weight).  ``out``: ``(dq, dk)``, which may be
    ``(dq_out, dk_out)``.  ``workspace``: a device tensor of ``bdlm_qk_rotate_workspace_bytes`` bytes (calls that may
    overlap in time need one each); allocated if not given and there is a weight."""
    c, n, H, KV, args = _inputs(rot, q, k, positions, q_weight, k_weight, eps)
    rdq, rdk = _as_long(c, "dq_out", dq_out, H, n), _as_long(c, "dk_out", dk_out, KV, n)
    out, rows = _out_rows(c, out, ("dq", "dk"), q, k, stream)
    dqw = dkw = dqw_at = dkw_at = at = None
    nbytes = 0
    if q_weight is not None or k_weight is not None:
        new = _made(stream, c.device, _new_weight_grads, *[w for w in (q_weight, k_weight) if w is not None])
        if q_weight is not None:
            dqw, dqw_at = new[0], new[0].data_ptr()
        if k_weight is not None:
            dkw, dkw_at = new[-1], new[-1].data_ptr()
        if c.workspace_bytes is None:
            c.workspace_bytes = lib().bdlm_qk_rotate_workspace_bytes(c.head_dim)
        workspace = _workspace(workspace, c.workspace_bytes, c.device, stream)
        at, nbytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _launch(c, stream, lib().bdlm_qk_rotate_bwd, *args, rdq, rdk, *rows, dqw_at, dkw_at, at, nbytes)
    return (*out, dqw, dkw)
