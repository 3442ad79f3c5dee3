"""The weights' gradients of rotation over many rows: a lane's sums stay short.

Rows are alike, so that every lane's sum is off the same way and nothing averages out.  At position 0 nothing turns, so
with r = 1 / sqrt(mean x^2 + eps) an element's gradient is (rows x heads) times the heads' mean of dy x r.  Bound: the
terms' own error (r's, ``rotate_oracle.normed``, and 2 v for the product's factors), at most 64 of them added in fp32 by
a lane, 6 steps for the wave's lanes and the workgroup's waves (12 with their sums' rounding), what is added after in 64
bits, and the result's rounding (v = 2^-24).
"""
import pytest
import torch

import paper_2609_19242_amd as bd
from tests import rotate_oracle

pytestmark = pytest.mark.gpu
DEV, BF, F32 = "cuda", torch.bfloat16, torch.float32
V = 2.0 ** -24


# 16 heads: a lane adds up 512 to 1,024 products; a row of many heads: one wave adds up hundreds of one row's
@pytest.mark.parametrize("dtype,n,H", [(BF, 1 << 21, 16), (F32, 1 << 20, 16), (BF, 1000, 70001), (F32, 3, 1 << 22)])
def test_long_sums(dtype, n, H):
    D, rot = 64, bd.rotary(64)
    g = torch.Generator().manual_seed(H)
    x, dy = (torch.randn(2, D, generator=g).to(dtype).to(DEV) for _ in range(2))
    w = torch.ones(D, dtype=dtype, device=DEV)
    q, k = (x[i].expand(n, h, D).contiguous() for i, h in enumerate((H, 1)))
    d = [dy[i].expand(n, h, D).contiguous() for i, h in enumerate((H, 1))]
    pos = torch.zeros(n, dtype=torch.int32, device=DEV)
    got = bd.qk_rotate_bwd(rot, q, k, pos, *d, w, w, eps=1e-6, out=tuple(d))[2:]
    torch.cuda.synchronize()
    for i, h in enumerate((H, 1)):
        r, _, er = rotate_oracle.normed(x[i].cpu().double(), 1.0, 1e-6, dtype)
        dw = n * h * (dy[i].cpu().double() * x[i].cpu().double() * r)
        e = (got[i].cpu().double() - dw).abs() / dw.abs()
        print(f"{'qk'[i]}: {float(e.max()) / V:.1f} steps", flush=True)
        assert float(e.max()) <= 1.05 * (er + (2 + 64 + 12 + 1) * V)
