"""64-bit oracle of packed attention and of attention over a paged cache, and how far a kernel may be off.

Plain loops over sequences and heads in float64 on the CPU, from the definitions.  ``bound`` holds, per element, what
the kernels' roundings can add up to (u is half a step, relative: 2^-8 in bf16, 2^-24 in fp32):
  P carries e_p = 2^-24 |LSE| (LSE saved in fp32) + 2^-17 in the bf16 path (scores summed in fp32 over d = 128 products
  of unit size: 128 * 2^-24, and the exponential's 2^-22), or 2^-40 in the fp32 path (all in 64 bits);
  the softmax scale is an fp32 number: 1 / sqrt(128) is off by up to u32 = 2^-24 of itself, so a score s by u32 |s| and
  P = exp(s - LSE) by u32 (|s| + the row's largest |s|), the second part through LSE, a mean of the row's scores (this
  makes up the whole error of the fp32 path at d = 128, which the other terms, without it, put too low);
  the bf16 path rounds P and dS to bf16 before the second products (u each) and reads the rounded O for D;
  every output is rounded once (u).  Second-order terms: factor 1.05.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def visible(nq, nk, block, window):
    """[nq][nk] truth values: row i is at position nk - nq + i."""
    x = (torch.arange(nq) + (nk - nq))[:, None]
    j = torch.arange(nk)[None]
    e = torch.div(x, block, rounding_mode="floor") * block + block
    vis = (j < e) & (x >= 0)
    if window:
        vis &= j >= e - window
    return vis


def head(q, k, v, vis, scale, dtype, do=None):
    """One head in float64: {name: (value, bound)} of o, lse and, with do, dq, dk, dv."""
    u, exact = U[dtype], dtype == torch.float32
    prod = 0.0 if exact else u  # P and dS are rounded before their products
    s = (q @ k.T) * scale
    s = torch.where(vis, s, torch.tensor(-math.inf, dtype=torch.float64))
    if k.shape[0]:
        z = torch.logsumexp(s, 1)
    else:
        z = torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
    p = torch.where(vis, torch.exp(s - torch.where(z == -math.inf, 0.0, z)[:, None]), 0.0)
    kk, vv = (torch.where(vis.any(0)[:, None], t, 0.0) for t in (k, v))  # (rows that nobody sees may hold anything)
    o = p @ vv
    zabs = torch.where(z == -math.inf, 0.0, z.abs())[:, None]
    # scores: fp32 sums of d products of the rows' sizes
    ds_score = 0.0 if exact else 2.0 ** -24 * 16 * scale * (q.abs() @ kk.abs().T)
    sabs = torch.where(vis, s.abs(), 0.0)
    top = sabs.amax(1, keepdim=True) if s.shape[1] else 0.0
    e_p = 2.0 ** -24 * (zabs + sabs + top) + (2.0 ** -40 if exact else 2.0 ** -20 + ds_score)
    e_o = ((e_p + prod) * p) @ vv.abs()
    out = {"o": (o, 1.05 * (e_o + u * o.abs()) + 1e-30), "lse": (z, 2 ** -22 * (1 + zabs[:, 0]) + (0 if exact else 1e-5))}
    if do is None:
        return out
    do = torch.where(vis.any(1)[:, None], do, 0.0)
    dd = (do * o).sum(1, keepdim=True)
    ds = p * (do @ vv.T - dd)
    e_d = u * (do.abs() * o.abs()).sum(1, keepdim=True) + (do.abs() * e_o).sum(1, keepdim=True) + 2.0 ** -22 * dd.abs()
    e_dp = 0.0 if exact else 2.0 ** -24 * 16 * (do.abs() @ vv.abs().T)
    e_ds = e_p * ds.abs() + p * (e_d + e_dp) + prod * ds.abs()
    out["dq"] = (ds @ kk) * scale, e_ds @ kk.abs() * scale
    out["dk"] = (ds.T @ q) * scale, e_ds.T @ q.abs() * scale
    out["dv"] = p.T @ do, ((e_p + prod) * p).T @ do.abs()
    for n in ("dq", "dk", "dv"):
        ref, b = out[n]
        out[n] = ref, 1.05 * (b + u * ref.abs()) + 1e-30
    return out


def packed(q, k, v, seqs, scale=None, block=1, window=0, do=None):
    """Oracle of a packed call: seqs [(q_start, q_len, k_start, k_len)].  Returns {name: (value, bound)} of tensors
    shaped like the call's outputs; rows of no sequence are NaN."""
    H, KV, D = q.shape[1], k.shape[1], q.shape[2]
    scale = scale or 1.0 / math.sqrt(D)
    nan = lambda *s: torch.full(s, math.nan, dtype=torch.float64)  # noqa: E731
    shapes = {"o": q.shape, "lse": (H, q.shape[0])}
    if do is not None:
        shapes.update(dq=q.shape, dk=k.shape, dv=v.shape)
    out = {n: (nan(*s), nan(*s)) for n, s in shapes.items()}
    Q, K, V = (t.detach().cpu().double() for t in (q, k, v))
    dO = do.detach().cpu().double() if do is not None else None
    for q0, nq, k0, nk in seqs:
        vis = visible(nq, nk, block, window)
        for n in ("dk", "dv"):
            if n in out:
                for t in out[n]:
                    t[k0:k0 + nk] = 0
        for h in range(H):
            g = h // (H // KV)
            qs, ks = slice(q0, q0 + nq), slice(k0, k0 + nk)
            r = head(Q[qs, h], K[ks, g], V[ks, g], vis, scale, q.dtype, dO[qs, h] if do is not None else None)
            for i in range(2):
                out["o"][i][qs, h] = r["o"][i]
                out["lse"][i][h, qs] = r["lse"][i]
                if do is not None:
                    out["dq"][i][qs, h] = r["dq"][i]
                    out["dk"][i][ks, g] += r["dk"][i]
                    out["dv"][i][ks, g] += r["dv"][i]
    return out


def check(name, got, ref, bound):
    """got within bound of ref wherever ref is a number; -inf must match; NaN in ref: not looked at."""
    g = got.detach().double().cpu()
    assert g.shape == ref.shape, (name, g.shape, ref.shape)
    there = ~torch.isnan(ref)
    assert not torch.isnan(g[there]).any(), f"{name}: NaN at {torch.nonzero(torch.isnan(g) & there)[:4].tolist()}"
    inf = ref == -math.inf
    assert torch.equal((g == -math.inf) & there, inf), f"{name}: -inf pattern differs"
    d = torch.where(there & ~inf, (g - ref).abs() - bound, torch.tensor(-1.0, dtype=torch.float64))
    used = torch.where(there & ~inf & (bound > 1e-30), (g - ref).abs() / bound, torch.tensor(0.0, dtype=torch.float64))
    m = float(used.max()) if used.numel() else 0.0
    print(f"{name}: {m:.3f} of the bound", flush=True)
    assert not d.numel() or float(d.max()) <= 0, (name, float(d.max()), torch.nonzero(d == d.max())[0].tolist())
