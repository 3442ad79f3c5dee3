"""64-bit oracle of rotated queries and keys, and how far a kernel may be off.

Written from the definitions, on the CPU.  The bounds add up the kernels' roundings (v = 2^-24, half a step of fp32; u half
a step of the outputs' type):
  angle: position times frequency in 64 bits, three roundings of the product here or there: 2^-51 of the angle; in fp32 the
  rest of the turn (1 v), its factor pi / 2 (2 v of at most 0.8) and the series (2 v): a cosine or sine is off by at most
  E_t = 5 v + 2^-51 |t|;
  r: in bf16 calls the fp32 sum of squares (16 products and sums of a lane, up to 4 of the lanes: 20 v, half of it in the
  root), the mean and eps (2 v), and the root's 1 step (2 v): 14 v; in fp32 calls 64-bit sums, rounded: 2 v;
  n = x r w: 2 v more;  a turned element: E_t, 3 v for its two products and their sum.
"""
import math

import torch

V = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def angles(freqs, axes, positions):
    """[rows][1][pairs]"""
    p = positions.cpu().double()
    p = p[torch.tensor(axes)].T if p.dim() == 2 else p[:, None]
    return (p * torch.tensor(freqs, dtype=torch.float64))[:, None]


def turned(x, t, interleaved, back=False):
    dim = 2 * t.shape[-1]
    c, s = torch.cos(t), torch.sin(t)
    if back:
        s = -s
    y = x.clone()
    i = torch.arange(dim // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + dim // 2)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def pair_sizes(x, t, interleaved):
    """|n1| + |n2| of each element's pair, 0 for the elements that stay; and the angle's size."""
    dim = 2 * t.shape[-1]
    size, far = torch.zeros_like(x), torch.zeros_like(x)
    i = torch.arange(dim // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + dim // 2)
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    far[..., a] = far[..., b] = t.abs().expand(*x.shape[:-1], dim // 2)
    return size, far


def turn_error(n, en, t, interleaved):
    """Error of the turned elements, before they are rounded, of n off by en."""
    size, far = pair_sizes(n, t, interleaved)
    size_en, _ = pair_sizes(en, t, interleaved)
    inside = size_en + (8 * V + 2.0 ** -51 * far) * size
    return torch.where(far + size_en + size > 0, inside, en)


def normed(x, w, eps, dtype):
    """r, n and r's relative error."""
    if eps is None:
        return torch.ones_like(x[..., :1]), x, 0.0
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return r, x * r * w, (14 if dtype == torch.bfloat16 else 2) * V


def forward(x, w, t, eps, interleaved):
    """(y, bound) of a tensor [rows][heads][D]."""
    dtype, x = x.dtype, x.cpu().double()
    w = torch.ones(x.shape[-1], dtype=torch.float64) if w is None else w.cpu().double()
    r, n, er = normed(x, w, eps, dtype)
    y = turned(n, t, interleaved)
    e = turn_error(n, (er + (2 * V if eps is not None else 0.0)) * n.abs(), t, interleaved)
    return y, 1.05 * (e + U[dtype] * y.abs()) + 1e-37


def backward(x, w, t, eps, interleaved, dy):
    """{dx: (value, bound), dw: (value, bound)}"""
    dtype, x, dy = x.dtype, x.cpu().double(), dy.cpu().double()
    D = x.shape[-1]
    w = torch.ones(D, dtype=torch.float64) if w is None else w.cpu().double()
    g = turned(dy, t, interleaved, back=True)
    eg = turn_error(dy, torch.zeros_like(dy), t, interleaved)
    if eps is None:
        return {"dx": (g, 1.05 * (eg + U[dtype] * g.abs()) + 1e-37)}
    r, _, er = normed(x, w, eps, dtype)
    xh, h = x * r, g * w
    m = (h * xh).mean(-1, keepdim=True)
    dx = r * (h - xh * m)
    eh = w.abs() * eg + V * h.abs()
    # the mean: its terms, their sum (as for r) and its factors
    sums = (24 if dtype == torch.bfloat16 else 4) * V + er
    em = (eh * xh.abs()).mean(-1, keepdim=True) + sums * (h * xh).abs().mean(-1, keepdim=True)
    edx = r * (eh + xh.abs() * em + (er * 2 + 4 * V) * (h.abs() + xh.abs() * m.abs()))
    # a lane adds up to 64 products of the tests' sizes, then 16 lanes, 4 waves and the workgroups
    terms = (g * xh).abs()
    dw = (g * xh).sum((0, 1))
    edw = (eg * xh.abs() + (er + 2 * V) * terms).sum((0, 1)) + 76 * V * terms.sum((0, 1)) + V * dw.abs()
    return {"dx": (dx, 1.05 * (edx + U[dtype] * dx.abs()) + 1e-37), "dw": (dw, 1.05 * edw + 1e-37)}
