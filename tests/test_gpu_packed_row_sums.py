"""dQ of rows whose keys all lie in one tile of 64: sum_j dS_ij = 0 there as far as P's sum is 1, because D comes from
the tile's own products, also where the whole tile is seen by every row (blocks of 64, texts of one block).

V is a large row plus small steps, K a large row plus noise: dP - D is then small against dP, and an error of D common
to a row, which a D formed from the bf16 O has (2^-8 |dO||O|), shows in dQ as that much of the large row.

Bound of dQ, from the bf16 path's roundings without that term, u = 2^-8: P is off by e_p = 2^-24 (2 |LSE| + |s| + top) +
2^-20 + 2^-20 scale |q||k| of itself (as in serving_util), dS is rounded to bf16 (u |dS|), dP - D is a sum of 64 to 128
products in fp32 on top of -D (2^-20 |dO||v| + 2^-24 |D|), twice for what the row's own correction adds, and D's own
error of up to u (|dO||O|) is left over to the extent that the P of the tile do not add up to 1: e_p of it.  The output
is rounded once."""
import math

import pytest
import torch

import paper_2609_19242_amd as bd
import synth
from tests.serving_util import visible

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
U = 2.0 ** -8


@pytest.mark.parametrize("H,KV", [(2, 2), (4, 2), (8, 2), (3, 1)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ql,kl,block,window", [
    ([64, 64], [64, 64], 64, 0),          # texts of one block
    ([256, 100], [256, 100], 64, 64),     # the keys of a row's own block
    ([300], [300], 64, 0),                # the first block of a longer text
    ([50, 32], [50, 64], 128, 0),         # less than a tile; the last rows of a tile
    ([40, 7, 130], [40, 71, 130], 1, 20)  # tiles that rows see in part
])
def test_rows_with_all_their_keys_in_one_tile(ql, kl, block, window, H, KV, D):
    nq, nk = sum(ql), sum(kl)
    q, do = (synth.normal((nq, H, D), 71 + i, BF) for i in range(2))
    k = (4 * synth.normal((1, KV, D), 73, torch.float32) + synth.normal((nk, KV, D), 74, torch.float32) / 8).to(BF)
    v = (2 + synth.normal((1, KV, D), 75, torch.float32) / 4 + synth.normal((nk, KV, D), 76, torch.float32) / 32).to(BF)
    plan = bd.packed_plan(ql, kl, heads=H, kv_heads=KV, head_dim=D, dtype=BF, block_size=block, window=window)
    dev = [t.cuda() for t in (q, k, v)]
    o, lse = bd.packed_fwd(plan, *dev)
    dq = bd.packed_bwd(plan, *dev, o, lse, do.cuda())[0].cpu().double()
    q, k, v, do = (t.double() for t in (q, k, v, do))
    scale, worst, rows, q0, k0 = 1 / math.sqrt(D), 0.0, 0, 0, 0
    for n, m in zip(ql, kl):
        vis = visible(n, m, block, window)
        first, last = vis.int().argmax(1), m - 1 - vis.flip(1).int().argmax(1)
        one = vis.any(1) & (first // 64 == last // 64)
        rows += int(one.sum())
        for h in range(H):
            Q, dO, K, V = q[q0:q0 + n, h], do[q0:q0 + n, h], k[k0:k0 + m, h // (H // KV)], v[k0:k0 + m, h // (H // KV)]
            s = (Q @ K.T * scale).masked_fill(~vis, -math.inf)
            z = torch.logsumexp(s, 1, keepdim=True)
            p = torch.exp(s - z).masked_fill(~vis, 0.0)
            dp, O = dO @ V.T, p @ V
            dd = (dO * O).sum(1, keepdim=True)
            ds = p * (dp - dd)
            sa = s.masked_fill(~vis, 0.0).abs()
            e_p = 2.0 ** -24 * (2 * z.abs() + sa + sa.amax(1, keepdim=True)) + 2.0 ** -20 * (
                1 + scale * (Q.abs() @ K.abs().T))
            e_p = e_p.masked_fill(~vis, 0.0)
            e_d = U * (dO.abs() * O.abs()).sum(1, keepdim=True) * e_p.amax(1, keepdim=True)
            e_dp = 2 * (2.0 ** -20 * (dO.abs() @ V.abs().T) + 2.0 ** -24 * dd.abs()) + e_d
            e_ds = (e_p + U) * ds.abs() + p * (e_dp + (e_p * ds.abs()).sum(1, keepdim=True))
            ref = ds @ K * scale
            bound = 1.05 * (e_ds @ K.abs() * scale + U * ref.abs()) + 1e-30
            used = ((dq[q0:q0 + n, h] - ref).abs() / bound)[one]
            worst = max(worst, float(used.max()) if len(used) else 0.0)
        q0, k0 = q0 + n, k0 + m
    print(f"{rows} rows: {worst:.3f} of the bound", flush=True)
    assert rows > 0 and worst <= 1
