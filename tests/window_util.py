"""64-bit oracle of attention with a sliding window and first tokens that stay visible, packed and over a paged cache.

The formulas and bounds of a head are ``serving_util.head``'s, over the visible pairs of this rule: row at position x,
e = block * (floor(x / block) + 1), sees j < e with j >= e - window (window 0: all) or j < sinks.
"""
import math

import torch

from tests.serving_util import head


def visible(nq, nk, block=1, window=0, sinks=0):
    """[nq][nk] truth values, one pair at a time: row i is at position nk - nq + i."""
    vis = torch.zeros(nq, nk, dtype=torch.bool)
    for i in range(nq):
        x = nk - nq + i
        if x < 0:
            continue
        e = block * (x // block + 1)
        lo = max(0, e - window) if window else 0
        vis[i, :min(sinks, e, nk)] = True
        vis[i, min(lo, nk):min(e, nk)] = True
    return vis


def nan(*s):
    return torch.full(s, math.nan, dtype=torch.float64)


def packed(q, k, v, seqs, scale=None, block=1, window=0, sinks=0, do=None):
    """{name: (value, bound)} of a packed call over seqs [(q_start, q_len, k_start, k_len)]; rows of no sequence are NaN."""
    H, KV, D = q.shape[1], k.shape[1], q.shape[2]
    scale = scale or 1.0 / math.sqrt(D)
    shapes = {"o": q.shape, "lse": (H, q.shape[0])}
    if do is not None:
        shapes.update(dq=q.shape, dk=k.shape, dv=v.shape)
    out = {n: (nan(*s), nan(*s)) for n, s in shapes.items()}
    Q, K, V = (t.detach().cpu().double() for t in (q, k, v))
    dO = do.detach().cpu().double() if do is not None else None
    for q0, nq, k0, nk in seqs:
        vis = visible(nq, nk, block, window, sinks)
        qs, ks = slice(q0, q0 + nq), slice(k0, k0 + nk)
        for n in ("dk", "dv"):
            if n in out:
                for t in out[n]:
                    t[ks] = 0
        for h in range(H):
            g = h // (H // KV)
            r = head(Q[qs, h], K[ks, g], V[ks, g], vis, scale, q.dtype, dO[qs, h] if do is not None else None)
            for i in range(2):
                out["o"][i][qs, h], out["lse"][i][h, qs] = r["o"][i], r["lse"][i]
                if do is not None:
                    out["dq"][i][qs, h] = r["dq"][i]
                    out["dk"][i][ks, g] += r["dk"][i]
                    out["dv"][i][ks, g] += r["dv"][i]
    return out
