"""Packed attention, forward and backward, against the 64-bit oracle: every type and head layout, lengths from none to
several tiles, more queries than keys and fewer, blocks, windows, strided inputs and outputs, gaps."""
import math

import pytest
import torch

import paper_2609_19242_amd as bd
import synth
from tests.serving_util import check, packed, visible

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def rows_of(lens, gap=0):
    out, at = [], 0
    for n in lens:
        out.append(at)
        at += n + gap
    return out, at


def run(ql, kl, H, KV, D, dtype, block=1, window=0, gap=0, scale=0.0, fused=False, backward=True, seed=0):
    qs, nq = rows_of(ql, gap)
    ks, nk = rows_of(kl, gap)
    nq, nk = nq + 3, nk + 3  # rows behind the last sequence
    if fused:
        assert ql == kl
        qkv = synth.normal((nq, H + 2 * KV, D), seed, dtype).to(DEV)
        q, k, v = qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:]
    else:
        q = synth.normal((nq, H, D), seed, dtype).to(DEV)
        k, v = (synth.normal((nk, KV, D), seed + i, dtype).to(DEV) for i in (1, 2))
    do = synth.normal((nq, H, D), seed + 3, dtype).to(DEV)
    # what lies between the sequences is nobody's: NaN there must not be seen
    for t, st, ln in ((q, qs, ql), (k, ks, kl), (v, ks, kl), (do, qs, ql)):
        mine = torch.zeros(t.shape[0], dtype=torch.bool)
        for a, n in zip(st, ln):
            mine[a:a + n] = True
        if not (fused and t is not do):
            t[~mine.to(DEV)] = math.nan
    plan = bd.packed_plan(ql, kl, heads=H, kv_heads=KV, head_dim=D, dtype=dtype, block_size=block, window=window,
                          scale=scale, q_starts=qs, k_starts=ks)
    new = lambda t, stride=None: torch.full(t, 7.0, dtype=dtype, device=DEV)  # noqa: E731
    o, lse = new((nq, H, D)), torch.full((H, nq), 7.0, device=DEV)
    bd.packed_fwd(plan, q, k, v, out=(o, lse))
    ref = packed(q, k, v, list(zip(qs, ql, ks, kl)), scale=scale or None, block=block, window=window,
                 do=do if backward else None)
    got = {"o": o, "lse": lse}
    if backward:
        if fused:
            dqkv = new((nq, H + 2 * KV, D))
            grads = dqkv[:, :H], dqkv[:, H:H + KV], dqkv[:, H + KV:]
        else:
            grads = new((nq, H, D)), new((nk, KV, D)), new((nk, KV, D))
        bd.packed_bwd(plan, q, k, v, o, lse, do, out=grads)
        got.update(zip(("dq", "dk", "dv"), grads))
    torch.cuda.synchronize()
    for n, t in got.items():
        check(n, t, *ref[n])
        untouched = torch.isnan(ref[n][0])
        assert torch.all(t.cpu()[untouched] == 7.0), f"{n}: rows of no sequence were written"
    return got


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,KV,D", [(4, 2, 128), (4, 4, 64), (6, 2, 128), (8, 1, 64), (3, 3, 128)])
def test_lengths(H, KV, D, dtype):
    run([1, 0, 129, 17, 64, 200], [1, 0, 129, 17, 64, 200], H, KV, D, dtype, seed=3)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("ql,kl", [([1], [1]), ([1, 1, 1], [257, 64, 5]), ([5, 70, 131], [300, 70, 0]),
                                   ([90, 260, 33], [40, 3, 32]), ([0, 9], [130, 9]), ([0], [0])])
def test_queries_are_the_last_tokens(ql, kl, dtype):
    run(ql, kl, 4, 2, 128, dtype, seed=5)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block,window", [(32, 0), (7, 0), (1, 1), (1, 50), (16, 40), (24, 5), (500, 0), (3, 100000)])
def test_blocks_and_windows(block, window, dtype):
    run([150, 33, 260], [150, 80, 200], 4, 2, 64, dtype, block=block, window=window, seed=7)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,KV,D", [(4, 2, 128), (3, 1, 64)])
def test_fused_projection(H, KV, D, dtype):
    run([60, 130, 1], [60, 130, 1], H, KV, D, dtype, fused=True, seed=9)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_gaps_are_left_alone(dtype):
    run([40, 1, 129], [70, 128, 129], 4, 2, 128, dtype, gap=11, seed=11)


def test_scale():
    run([100, 30], [100, 30], 4, 2, 128, BF, scale=0.5, seed=13)


def test_long_sequences_with_cut_walks():
    run([900, 30, 1100], [900, 700, 1100], 2, 1, 128, BF, seed=15)


def test_many_sequences_fill_the_card():
    ql = [1 + (37 * i) % 140 for i in range(150)]
    run(ql, ql, 8, 4, 64, BF, backward=False, seed=17)


def test_same_bits_twice_and_in_another_packing():
    """A sequence's results do not depend on where it lies (its tiles walk alike whatever the others are)."""
    a = run([140, 60], [140, 60], 4, 2, 128, BF, seed=19, backward=False)
    b = run([140, 60], [140, 60], 4, 2, 128, BF, seed=19, backward=False)
    assert torch.equal(a["o"], b["o"]) and torch.equal(a["lse"], b["lse"])


def test_one_sequence_equals_the_joint_call_on_its_clean_half():
    L, H, KV, D = 384, 4, 2, 128
    q, k, v = (synth.normal((L, h, D), 20 + i, BF).to(DEV) for i, h in enumerate((H, KV, KV)))
    plan = bd.packed_plan([L], heads=H, kv_heads=KV, head_dim=D, dtype=BF)
    o, lse = bd.packed_fwd(plan, q, k, v)
    p = bd.make_problem(1, L, 1, H, KV, D, BF)
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    r = bd.Range(bd.CLEAN, 0, L)
    bd.attn_partial_fwd(p, r, q, o2, lse2, r, k, v)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_graph_replays():
    H, KV, D = 4, 2, 128
    ql = [100, 7, 260]
    n = sum(ql)
    q, k, v, do = (synth.normal((n, h, D), 30 + i, BF).to(DEV) for i, h in enumerate((H, KV, KV, H)))
    plan = bd.packed_plan(ql, heads=H, kv_heads=KV, head_dim=D, dtype=BF)

    def step():
        o, lse = bd.packed_fwd(plan, q, k, v)
        return (o, lse) + bd.packed_bwd(plan, q, k, v, o, lse, do)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = step()
    for i in range(4):
        q.copy_(synth.normal(q.shape, 50 + i, BF))
        g.replay()
        torch.cuda.synchronize()
        eager = step()
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    H, KV, D = 4, 2, 64
    ql = [300, 41]
    plan = bd.packed_plan(ql, heads=H, kv_heads=KV, head_dim=D, dtype=BF)
    ins = [[synth.normal((sum(ql), h, D), 60 + 10 * j + i, BF).to(DEV) for i, h in enumerate((H, KV, KV, H))]
           for j in range(2)]
    want = []
    for q, k, v, do in ins:
        o, lse = bd.packed_fwd(plan, q, k, v)
        want.append((o, lse) + bd.packed_bwd(plan, q, k, v, o, lse, do))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ins]
    got = []
    for s, (q, k, v, do) in zip(streams, ins):
        with torch.cuda.stream(s):
            o, lse = bd.packed_fwd(plan, q, k, v)
            got.append((o, lse) + bd.packed_bwd(plan, q, k, v, o, lse, do))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("ql,kl,block,window", [([20, 33], [300, 170], 1, 40), ([1, 5, 64], [129, 400, 200], 1, 1),
                                                ([40, 100], [400, 333], 16, 70), ([10], [200], 64, 10)])
def test_keys_that_no_row_sees_may_hold_anything(ql, kl, block, window, what, dtype):
    """The past that a window has left behind: its keys and values, evicted or never written."""
    H, KV, D = 4, 2, 64
    qs, nq = rows_of(ql)
    ks, nk = rows_of(kl)
    q, do = (synth.normal((nq, H, D), 70 + i, dtype).to(DEV) for i in range(2))
    k, v = (synth.normal((nk, KV, D), 80 + i, dtype).to(DEV) for i in range(2))
    for s, (a, n, m) in enumerate(zip(ks, ql, kl)):
        seen = visible(n, m, block, window).any(0).to(DEV)
        assert not seen.all()
        for t in (k, v):
            t[a:a + m][~seen] = what
    plan = bd.packed_plan(ql, kl, heads=H, kv_heads=KV, head_dim=D, dtype=dtype, block_size=block, window=window)
    o, lse = bd.packed_fwd(plan, q, k, v)
    dq, dk, dv = bd.packed_bwd(plan, q, k, v, o, lse, do)
    torch.cuda.synchronize()
    ref = packed(q, k, v, list(zip(qs, ql, ks, kl)), block=block, window=window, do=do)
    for n, t in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        check(n, t, *ref[n])


def test_padded_batch():
    """[batch][longest] rows with lengths: the padding is read and written by nobody."""
    B, S, H, KV, D = 3, 150, 4, 2, 64
    lens = [150, 1, 77]
    q, do = (synth.normal((B * S, H, D), 90 + i, BF).to(DEV) for i in range(2))
    k, v = (synth.normal((B * S, KV, D), 95 + i, BF).to(DEV) for i in range(2))
    starts = [b * S for b in range(B)]
    for b, n in enumerate(lens):
        for t in (q, k, v, do):
            t[b * S + n:(b + 1) * S] = math.nan
    plan = bd.packed_plan(lens, heads=H, kv_heads=KV, head_dim=D, dtype=BF, q_starts=starts)
    out = torch.zeros_like(q), torch.zeros(H, B * S, device=DEV)
    o, lse = bd.packed_fwd(plan, q, k, v, out=out)
    grads = tuple(torch.zeros_like(t) for t in (q, k, v))
    bd.packed_bwd(plan, q, k, v, o, lse, do, out=grads)
    torch.cuda.synchronize()
    ref = packed(q, k, v, [(s, n, s, n) for s, n in zip(starts, lens)], do=do)
    for n, t in zip(("o", "lse", "dq", "dk", "dv"), (o, lse) + grads):
        check(n, t, *ref[n])
        assert not torch.isnan(t).any()


@pytest.mark.parametrize("other", [False, True])
def test_new_outputs_hold_zeros_in_rows_of_no_sequence(other):
    q, k, v, do = (synth.normal((40, h, 64), 60 + i, BF).to(DEV) for i, h in enumerate((4, 2, 2, 4)))
    stream = torch.cuda.Stream() if other else None
    for starts, n in (([0, 20], 40), (None, 40), (None, 27)):  # gaps, rows behind the last, neither
        plan = bd.packed_plan([10, 17], heads=4, kv_heads=2, head_dim=64, dtype=BF, q_starts=starts)
        for _ in range(2):  # (memory that held something)
            trash = [torch.full((n, h, 64), math.nan, dtype=BF, device=DEV) for h in (4, 4, 2, 2)]
            trash.append(torch.full((4, n), math.nan, device=DEV))
            del trash
            torch.cuda.synchronize()
            o, lse = bd.packed_fwd(plan, q[:n], k[:n], v[:n], stream=stream)
            dq, dk, dv = bd.packed_bwd(plan, q[:n], k[:n], v[:n], o, lse, do[:n], stream=stream)
            torch.cuda.synchronize()
        mine = torch.zeros(n, dtype=torch.bool)
        for a, m in zip(starts or (0, 10), (10, 17)):
            mine[a:a + m] = True
        for t in (o, dq, dk, dv):
            assert torch.all(t.cpu()[~mine] == 0) and bool(torch.isfinite(t).all())
        assert torch.all(lse.cpu()[:, ~mine] == -math.inf) and bool(torch.isfinite(lse.cpu()[:, mine]).all())


# Few query tiles with long walks: the walks are cut into chunks, whose partial outputs are joined.
@pytest.mark.parametrize("H,KV,D", [(4, 1, 128), (4, 2, 64), (3, 1, 128), (2, 2, 64)])
@pytest.mark.parametrize("ql,kl,block,window", [
    ([1], [2500], 1, 0), ([70, 1, 3], [2000, 1700, 0], 1, 0), ([200], [2300], 32, 0), ([130, 40], [2400, 20], 1, 1900),
    ([1800], [1700], 1, 0), ([65], [4000], 5000, 0), ([1600], [1500], 4000, 0)])
def test_few_rows_with_long_walks(ql, kl, block, window, H, KV, D):
    plan = bd.packed_plan(ql, kl, heads=H, kv_heads=KV, head_dim=D, dtype=BF, block_size=block, window=window)
    # (24 and 27 key tiles are left whole at head_dim 64, where the products take half as long and the partial outputs do not)
    assert plan.fwd_workspace_bytes > 0 or (D == 64 and ql in ([1800], [1600]))
    run(ql, kl, H, KV, D, BF, block=block, window=window, gap=5, seed=41)


def test_cut_walks_are_the_same_every_time_and_in_a_given_workspace():
    plan = bd.packed_plan([90, 5], [3000, 2500], heads=8, kv_heads=2, head_dim=128, dtype=BF)
    q, k, v = (synth.normal((n, h, 128), 70 + h, BF).to(DEV) for n, h in ((95, 8), (5500, 2), (5500, 2)))
    ws = torch.full((plan.fwd_workspace_bytes,), 0xff, dtype=torch.uint8, device=DEV)
    o, lse = bd.packed_fwd(plan, q, k, v)
    for w in (None, ws, ws):
        o1, lse1 = bd.packed_fwd(plan, q, k, v, workspace=w)
        assert torch.equal(o, o1) and torch.equal(lse, lse1)
    with pytest.raises(bd.BdlmError):
        bd.packed_fwd(plan, q, k, v, workspace=ws[:-256])
    ref = packed(q, k, v, [(0, 90, 0, 3000), (90, 5, 3000, 2500)])
    check("o", o, *ref["o"])
    check("lse", lse, *ref["lse"])


def test_a_plan_dropped_while_its_kernels_run_elsewhere():
    q, k, v = (synth.normal((4000, h, 128), 80 + h, BF).to(DEV) for h in (8, 2, 2))
    kw = dict(heads=8, kv_heads=2, head_dim=128, dtype=BF)
    o, lse = bd.packed_fwd(bd.packed_plan([4000], **kw), q, k, v)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = torch.zeros_like(o), torch.zeros_like(lse)
    torch.cuda.synchronize()
    for use in (dict(stream=side), dict(stream=side.cuda_stream)):
        plan = bd.packed_plan([4000], **kw)
        n = plan._items.numel()
        for _ in range(20):  # (the last of these still waits when the plan is dropped)
            bd.packed_fwd(plan, q, k, v, out=out, **use)
        del plan
        other = [torch.full((n,), 0xff, dtype=torch.uint8, device=DEV) for _ in range(8)]
        torch.cuda.synchronize()
        assert torch.equal(out[0], o) and torch.equal(out[1], lse)
        del other


def test_two_graphs_of_cut_walks_share_their_workspaces():
    H, KV, D = 8, 2, 128
    plans = [bd.packed_plan(ql, kl, heads=H, kv_heads=KV, head_dim=D, dtype=BF) for ql, kl in (([90, 5], [3000, 2500]),
                                                                                              ([40], [4000]))]
    assert all(p.fwd_workspace_bytes > 0 for p in plans)
    ws = torch.empty(max(max(p.fwd_workspace_bytes, p.workspace_bytes) for p in plans), dtype=torch.uint8, device=DEV)
    q, do = (synth.normal((95, H, D), 90 + i, BF).to(DEV) for i in range(2))
    k, v = (synth.normal((5500, KV, D), 92 + i, BF).to(DEV) for i in range(2))

    def step(p, w):
        o, lse = bd.packed_fwd(p, q, k, v, workspace=w)
        return (o, lse) + bd.packed_bwd(p, q, k, v, o, lse, do, workspace=w)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for p in plans:
            step(p, ws)
    torch.cuda.current_stream().wait_stream(s)
    graphs, outs = [], []
    for p in plans:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(step(p, ws))
    for i in range(3):
        q.copy_(synth.normal(q.shape, 95 + i, BF))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for p, out in zip(plans, outs):
            want = step(p, None)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("D", [64, 128])
def test_more_workgroups_than_cus_in_two_teams(D):
    ql = [1100, 130, 1]
    plan = bd.packed_plan(ql, heads=28, kv_heads=28, head_dim=D, dtype=BF)
    assert plan._record.teams == 2 and plan._record.q_items * 28 > 256
    run(ql, ql, 28, 28, D, BF, gap=3, backward=False, seed=47)
