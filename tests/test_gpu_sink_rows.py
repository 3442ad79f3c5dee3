"""Gradients of rows that see at most 64 keys, in bf16 calls with a window and sinks, wherever those keys lie.

Values share a large part (20 + noise), so that the D formed from the rounded O is off by much of dS: such rows must take
theirs from the products, D = sum_j P_ij dP_ij.  The bound is ``serving_util.head``'s with another error of D for them
(v = 2^-24): with e_p and e_dp the errors of P and dP there, D' the D of the rounded O and dev = |dP - D| + |D' - D|,
  D = D' + sum_j P_ij (dP_ij - D'):  sum_j p_ij (e_dp + (e_p + 66 v) dev_ij) + 2 v (|D| + |D' - D|)
(66 v: the sum of up to 64 products and the two halves; 2 v: D's own roundings).
"""
import math

import pytest
import torch

import paper_2609_19242_amd as bd
from tests import window_util
from tests.serving_util import check

pytestmark = pytest.mark.gpu
DEV, BF = "cuda", torch.bfloat16
U, V = 2.0 ** -8, 2.0 ** -24


def head(q, k, v, vis, scale, do):
    """{name: (value, bound)} of dq, dk and D's place in them, one head in float64."""
    s = torch.where(vis, (q @ k.T) * scale, torch.tensor(-math.inf, dtype=torch.float64))
    z = torch.logsumexp(s, 1)[:, None]
    z = torch.where(z == -math.inf, 0.0, z)  # (rows that see nothing)
    p = torch.where(vis, torch.exp(s - z), 0.0)
    o = p @ v
    sabs = torch.where(vis, s.abs(), 0.0)
    e_p = V * (z.abs() + sabs + sabs.amax(1, keepdim=True)) + 2.0 ** -20 + V * 16 * scale * (q.abs() @ k.abs().T)
    e_o = ((e_p + U) * p) @ v.abs()
    dp, dd = do @ v.T, (do * o).sum(1, keepdim=True)
    ds = p * (dp - dd)
    e_dp = V * 16 * (do.abs() @ v.abs().T)
    e_d = U * (do.abs() * o.abs()).sum(1, keepdim=True) + (do.abs() * e_o).sum(1, keepdim=True) + 4 * V * dd.abs()
    dev = (dp - dd).abs() + e_d
    few_d = (p * (e_dp + (e_p + 66 * V) * dev)).sum(1, keepdim=True) + 2 * V * (dd.abs() + e_d)
    few = vis.sum(1, keepdim=True) <= 64
    e_ds = e_p * ds.abs() + p * (torch.where(few, few_d, e_d) + e_dp) + U * ds.abs()
    out = {"dq": (ds @ k * scale, e_ds @ k.abs() * scale), "dk": (ds.T @ q * scale, e_ds.T @ q.abs() * scale)}
    return {n: (x, 1.05 * (b + U * x.abs()) + 1e-30) for n, (x, b) in out.items()}


def grads(ql, kl, H, KV, D, block, window, sinks, seed, spread=0.5):
    kl = kl or ql
    plan = bd.packed_plan(ql, kl, heads=H, kv_heads=KV, head_dim=D, dtype=BF, block_size=block, window=window, sinks=sinks)
    g = torch.Generator().manual_seed(seed)
    q, k, v, do = (torch.randn(n, h, D, generator=g) for n, h in ((sum(ql), H), (sum(kl), KV), (sum(kl), KV), (sum(ql), H)))
    q, k, v, do = (t.to(BF).to(DEV) for t in (q, k, 20 + spread * v, do))
    o, lse = bd.packed_fwd(plan, q, k, v)
    got = dict(zip(("dq", "dk"), bd.packed_bwd(plan, q, k, v, o, lse, do)[:2]))
    torch.cuda.synchronize()
    Q, K, VV, dO = (t.cpu().double() for t in (q, k, v, do))
    ref = {n: [torch.zeros(t.shape, dtype=torch.float64) for _ in range(2)] for n, t in got.items()}
    few, q0, k0 = 0, 0, 0
    for nq, nk in zip(ql, kl):
        vis = window_util.visible(nq, nk, block, window, sinks)
        few += int((vis.sum(1) <= 64).sum())
        a, b = slice(q0, q0 + nq), slice(k0, k0 + nk)
        for h in range(H):
            r = head(Q[a, h], K[b, h * KV // H], VV[b, h * KV // H], vis, D ** -0.5, dO[a, h])
            for i in range(2):
                ref["dq"][i][a, h] = r["dq"][i]
                ref["dk"][i][b, h * KV // H] += r["dk"][i]
        q0, k0 = q0 + nq, k0 + nk
    for n in got:
        check(n, got[n], *ref[n])
    return plan, few


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,KV", [(2, 2), (4, 2), (3, 1), (4, 1)])
@pytest.mark.parametrize("window,sinks", [(1, 1), (16, 4), (32, 4), (48, 4), (30, 34), (3, 61)])
def test_windows_of_few_keys(D, H, KV, window, sinks):
    _, few = grads([300, 41], None, H, KV, D, 1, window, sinks, seed=window + sinks)
    assert few == 341


@pytest.mark.parametrize("H,KV", [(2, 2), (4, 1)])
@pytest.mark.parametrize("ql,kl,block,window,sinks", [
    ([270], None, 64, 100, 5),           # the last block ends behind the sequence: its rows see 55 keys, those before 105
    ([700], None, 512, 40, 3),           # a tile over two blocks, whose windows lie 472 keys apart
    ([150], None, 8, 64, 4),             # 68 keys, but for the first block and the last
    ([33, 0, 7, 90], [500, 20, 7, 1000], 1, 40, 5),
    ([40, 6], [10, 9], 1, 3, 2),         # rows that see nothing in front
    ([300], None, 1, 64, 1)])            # 65 keys: as without sinks, from the rounded O
def test_blocks_and_lengths(H, KV, ql, kl, block, window, sinks):
    grads(ql, kl, H, KV, 64, block, window, sinks, seed=len(ql) + window)


@pytest.mark.parametrize("D", [64, 128])
def test_cut_walks(D):
    # a tile over two blocks of 1,024 tokens walks all keys between their windows, in chunks
    plan, few = grads([1100], [2048], 4, 1, D, 1024, 50, 6, seed=3)
    assert few == 1100 and plan._record.dq.slots > 0


def test_the_same_bits_again_and_in_a_graph():
    plan = bd.packed_plan([500, 3], heads=4, kv_heads=1, head_dim=64, dtype=BF, window=32, sinks=4)

    def make(seed):
        g = torch.Generator().manual_seed(seed)
        q, k, v, do = (torch.randn(503, h, 64, generator=g).to(BF).to(DEV) for h in (4, 1, 1, 4))
        return q, k, v, *bd.packed_fwd(plan, q, k, v), do

    sets = [make(s) for s in (9, 10, 11)]
    expect = [[t.clone() for t in bd.packed_bwd(plan, *s)] for s in sets]
    assert all(torch.equal(a, b) for a, b in zip(expect[0], bd.packed_bwd(plan, *sets[0])))
    static = [t.clone() for t in sets[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        bd.packed_bwd(plan, *static)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = bd.packed_bwd(plan, *static)
    for i in (1, 2, 0, 1):
        for dst, src in zip(static, sets[i]):
            dst.copy_(src)
        for t in got:
            t.fill_(math.nan)
        graph.replay()
        torch.randn(512, 512, device=DEV).sum().item()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, expect[i])), i
