"""fp32 attention over the cache takes the softmax scale as the fp32 number that it is and everything else in 64 bits, as
the fp32 forward: the LSE is the exact one rounded once (half a step, and 2^-40 for the sums in 64 bits), with one chunk
and with several, whatever its size."""
import math

import pytest
import torch

import paper_2609_19242_amd as bd
import synth
from tests.test_gpu_prefix import build, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,n,H,KV,D,spare", [([300, 170, 90], 2, 8, 2, 64, 0), ([1500, 700], 1, 8, 2, 64, 50),
                                                 ([400, 333], 3, 4, 4, 128, 0)])
@pytest.mark.parametrize("scale", [0.3, 0.7, 1.1])
def test_lse_is_rounded_once(lens, n, H, KV, D, spare, scale):
    c = build(lens, 0, 16, KV, D, torch.float32, 71, spare=spare)
    q = synth.normal((len(lens), n, H, D), 72, torch.float32)
    q[..., 0] = 8.0  # an offset of some hundred to all scores
    c.k[..., 0] = torch.where(torch.isnan(c.k[..., 0]), c.k[..., 0], 60.0)
    o, lse = bd.prefix_attn(q.cuda(), c, 0, i32(range(len(lens))), scale=scale)
    torch.cuda.synchronize()
    exact = float(torch.tensor(scale, dtype=torch.float32).double())
    table, k, Q, worst = c.table.cpu().long(), c.k[0].cpu().double(), q.double(), 0.0
    for r, m in enumerate(lens):
        kk = k[table[r, :-(-m // 16)]].reshape(-1, KV, D)[:m]
        vis = torch.arange(m)[None] <= m - n + torch.arange(n)[:, None]
        for h in range(H):
            z = torch.logsumexp((Q[r, :, h] @ kk[:, h // (H // KV)].T * exact).masked_fill(~vis, -math.inf), 1)
            got = lse[r, h].cpu()
            step = torch.nextafter(z.abs().float(), torch.tensor(math.inf)).double() - z.abs().float().double()
            worst = max(worst, float(((got.double() - z).abs() / (0.5 * step + 2.0 ** -40 * z.abs())).max()))
    print(f"LSE around {float(z.mean()):.0f}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1
