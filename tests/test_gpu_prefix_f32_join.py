"""fp32 attention over the cache with scores that share a large offset: the log-sum-exps of a row's chunks are then large
numbers that differ little, and what joins the chunks' outputs must not lose that difference.

The softmax scale is an fp32 number, off by u = 2^-24 of itself at most: a score s is off by u |s|, of which only the
differences within a row count for P, so P by u (max s - min s).  A chunk's output is kept in fp32 (u of |O_j| <= sum P
|V|), the joined one is rounded once (u |O|); everything else is in 64 bits.  Second-order terms: factor 1.05."""
import math

import pytest
import torch

import paper_2609_19242_amd as bd
import synth
from tests.test_gpu_prefix import build, i32

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
OFFSET = 500.0  # of every score


def parts_of(q, c, prefix):
    R, n, H, D = q.shape
    return bd.prefix_attn_workspace_bytes(q, c, prefix) // (R * n * H * (4 * D + 8))


@pytest.mark.parametrize("lens,prefix,n,H,KV,D,spare,least", [
    ([1500, 2100], 0, 1, 4, 2, 64, 2, 2), ([1500, 2100], 0, 1, 4, 2, 64, 600, 3), ([300, 170], 0, 2, 4, 2, 64, 0, 0),
    ([300, 1900], 0, 3, 4, 1, 128, 400, 2), ([2300 + 40 * r for r in range(10)], 2250, 1, 4, 2, 128, 3, 3),
    ([20000], 0, 1, 8, 8, 64, 2, 17)])
def test_chunks_joined_at_large_log_sum_exps(lens, prefix, n, H, KV, D, spare, least):
    c = build(lens, prefix, 16, KV, D, torch.float32, 61, spare=spare)
    q = synth.normal((len(lens), n, H, D), 62, torch.float32)
    q[..., :8] *= 0.25
    q[..., 8:] = 0
    q[..., 0] = OFFSET * math.sqrt(D) / 64
    q = q.cuda()
    c.k[..., 0] = torch.where(torch.isnan(c.k[..., 0]), c.k[..., 0], 64.0)
    o, lse = bd.prefix_attn(q, c, 0, i32(range(len(lens))), prefix)
    torch.cuda.synchronize()
    parts = parts_of(q, c, prefix)
    assert parts >= least and (least or parts == 0)
    table, k, v, Q = c.table.cpu().long(), c.k[0].cpu().double(), c.v[0].cpu().double(), q.cpu().double()
    worst = 0.0
    for r, m in enumerate(lens):
        pages = table[r, :-(-m // 16)]
        kk, vv = (x[pages].reshape(-1, KV, D)[:m] for x in (k, v))
        vis = torch.arange(m)[None] <= m - n + torch.arange(n)[:, None]
        for h in range(H):
            g = h // (H // KV)
            s = Q[r, :, h] @ kk[:, g].T / math.sqrt(D)
            s = s.masked_fill(~vis, -math.inf)
            assert float(s[vis].min()) > OFFSET - 10
            z = torch.logsumexp(s, 1, keepdim=True)
            p = torch.exp(s - z)
            ref, spread = p @ vv[:, g], (s.amax(1) - s.masked_fill(~vis, math.inf).amin(1))[:, None]
            bound = 1.05 * ((U * spread + U) * (p @ vv[:, g].abs()) + U * ref.abs()) + 1e-30
            used = float(((o[r, :, h].cpu().double() - ref).abs() / bound).max())
            worst = max(worst, used)
            assert float((lse[r, h].cpu().double() - z[:, 0]).abs().max()) <= 2.1 * U * float(z.abs().max())
    print(f"{parts} parts: {worst:.3f} of the bound", flush=True)
    assert worst <= 1
